"""What the operators promise beyond their formulas' plain cases: streams, autograd's
bookkeeping, extreme magnitudes, and accuracy bounds column by column.

u = 2^-24 is float32's unit roundoff, 2^-8 bfloat16's; tolerances are worst cases
of the arithmetic, derived where they stand.
"""
import math

import pytest
import torch

from paper_2608_05088_amd import libmalt as lm

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lm.lib()


@pytest.fixture(scope="module")
def ops():
    from paper_2608_05088_amd import ops as module
    return module


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(seed, *shape, scale=1.0, dtype=F32):
    return (torch.randn(shape, device="cuda", generator=gen(seed)) * scale).to(dtype)


def turned(x):
    """x, its last two dimensions lying the other way round."""
    return x.transpose(-1, -2).contiguous().transpose(-1, -2)


def apart(x):
    """A vector whose elements lie two apart."""
    return torch.stack([x, x], -1)[..., 0]


def test_strided_inputs_on_another_stream(ops):
    """A call on a given stream waits for that stream alone, its layout copies too: the current one is busy meanwhile."""
    ids = torch.randint(0, 500, (30, 100), device="cuda", generator=gen(1))
    table, grad = randn(2, 500, 96), randn(3, 30, 100, 96)
    z, a = randn(4, 4, 5, 3001, scale=3.0, dtype=BF16), randn(5, 4, 5, 8, dtype=BF16)
    top = torch.randint(0, 3001, (4, 5, 8), device="cuda", generator=gen(6))
    y, w = torch.randint(0, 3001, (4, 5), device="cuda", generator=gen(7)), randn(8, 4, 5)
    y2, w2 = apart(y), apart(w)
    x, weight = randn(9, 3, 20, 300), randn(10, 90, 300)
    values, scales = ops.fp8_quantize_weight(weight)
    kw = dict(tau=2.0, alpha=0.5)
    calls = [lambda f, s: (ops.embedding(f(ids), f(table), **s),),
             lambda f, s: (ops.embedding_grad(f(ids), f(grad), 500, **s),),
             lambda f, s: (ops.distill_loss(f(z), f(a), f(top), f(y), **kw, **s),),
             lambda f, s: ops.distill_step(f(z), f(a), f(top), f(y), grad=f(w), **kw, **s),
             lambda f, s: ops.distill_step(f(z), f(a), f(top), y2, grad=w2, **kw, **s),
             lambda f, s: (ops.fp8_linear(f(x), f(weight), **s),),
             lambda f, s: (ops.fp8_linear(f(x), f(weight.t()), transposed=True, **s),),
             lambda f, s: (ops.fp8_forward(f(x), values, scales, **s),),
             lambda f, s: (ops.fp8_forward(f(x[:, :4]), values, scales, **s),),
             lambda f, s: tuple(t.view(torch.uint8) for t in ops.fp8_quantize_weight(f(weight), **s))]
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda._sleep(1000)
    start.record()
    torch.cuda._sleep(10_000_000)
    end.record()
    torch.cuda.synchronize()
    busy = int(10_000_000 * 100 / start.elapsed_time(end))   # 100 ms
    side = torch.cuda.Stream()
    for i, call in enumerate(calls):
        want = call(lambda t: t, {})
        laid = {}
        call(lambda t: laid.setdefault(len(laid), turned(t)), {})   # the inputs, before the streams part
        torch.cuda.synchronize()
        met = iter(laid.values())
        torch.cuda._sleep(busy)
        still = torch.cuda.Event()
        still.record()
        got = call(lambda t: next(met), dict(stream=side))
        side.synchronize()
        assert not still.query(), i
        with torch.cuda.stream(side):
            same = [torch.equal(p, q) for p, q in zip(got, want)]
        torch.cuda.synchronize()
        assert all(same), i


def test_a_backward_pass_refuses_what_was_written_over(ops):
    """Logits saved by the differentiable loss and then replaced by their gradient in place."""
    z, labels = randn(20, 6, 300).requires_grad_(), torch.arange(6, device="cuda")
    h = z * 1.0
    loss = ops.distill_loss(h, None, None, labels, alpha=1.0).sum()
    ops.distill_step(h, None, None, labels, alpha=1.0, out=h.detach())
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    table = randn(21, 10, 8).requires_grad_()
    h = table * 1.0
    square = (h * h).sum()
    ops.embedding_grad(labels, randn(22, 6, 8), 10, out=h.detach(), accumulate=True)
    with pytest.raises(RuntimeError, match="inplace"):
        square.backward()
