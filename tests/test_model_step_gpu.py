"""The operators together, as a training step and a serving step use them: norms with the residual's
addition, 8-bit layers, the head's loss and AdamW."""
import copy

import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu(stream_rounds):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_05088_amd import libmalt as lm
    lm.lib()


@pytest.fixture(scope="module")
def ops():
    from paper_2608_05088_amd import ops as module
    return module


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _plain_norm(x, w, eps=1e-6):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w


def _weights(seed, v, k):
    g = gen(seed)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    return dict(table=r(v, k) * 0.5, up=r(4 * k, k) / k ** 0.5, down=r(k, 4 * k) / (2 * k ** 0.5), n1=1 + 0.1 * r(k), n2=1 + 0.1 * r(k))


def test_a_training_step_in_float32(ops):
    """Table, norm, layers, residual and norm, head and AdamW: every gradient and every stepped parameter against the
    same in 64 bits.  Relative to each tensor's norm: sums of a few hundred float32 terms in a chain of six operators,
    6 x 300 x 2^-24 = 1e-4 at the worst."""
    v, k, n = 300, 96, 50
    w = {name: t.requires_grad_() for name, t in _weights(1, v, k).items()}
    ids = torch.randint(0, v, (n,), device="cuda", generator=gen(2))
    labels = torch.roll(ids, -1)
    labels[::7] = -100

    def layers(p, table, norm, norm_residual, head):
        h = table(ids, p["table"])
        a = norm(h, p["n1"])
        b = torch.nn.functional.gelu(a @ p["up"].t()) @ p["down"].t()
        y, s = norm_residual(b, p["n2"], h)
        return head(y, p["table"]) + 1e-3 * (s * s).sum()

    loss = layers(w, ops.embedding, ops.rms_norm, lambda x, g, r: ops.rms_norm(x, g, residual=r),
                  lambda y, t: ops.linear_cross_entropy(y, t, labels).sum())
    grads = torch.autograd.grad(loss, list(w.values()))
    w64 = {name: t.detach().double().requires_grad_() for name, t in w.items()}
    want = layers(w64, lambda i, t: t[i], _plain_norm, lambda x, g, r: (_plain_norm(x + r, g), x + r),
                  lambda y, t: torch.nn.functional.cross_entropy(y @ t.t(), labels, reduction="sum", ignore_index=-100))
    exact = torch.autograd.grad(want, list(w64.values()))
    assert abs(float(loss) - float(want)) <= 1e-4 * float(want)
    for (name, _), a, b in zip(w.items(), grads, exact):
        assert float((a - b).norm()) <= 1e-4 * float(b.norm()), name
    params = [t.detach() for t in w.values()]
    before = [p.clone() for p in params]
    states = [ops.adamw_state(p, 8 if p.numel() >= 4096 else 32) for p in params]
    ops.adamw_step(params, list(grads), states, lr=1e-3, betas=(0.9, 0.95), step=1, seed=3)
    for p, q, g in zip(params, before, grads):
        # A first step moves by lr in the gradient's sign wherever the gradient is far above eps.
        moved = q * (1 - 1e-3 * 0.01) - 1e-3 * g / (g.abs() + 1e-8)
        assert float((p - moved).abs().max()) <= 1e-3 * 1e-5 + 4 * 2.0 ** -24 * float(q.abs().max())


def test_a_token_through_8_bit_layers(ops):
    """Serving: the norm into 8 bits and kept 8-bit weights give the bits that the separate operators give."""
    k = 256
    w = _weights(4, 500, k)
    up = ops.fp8_quantize_weight(w["up"])
    for n in (1, 5, 40):
        h, b = torch.randn((n, k), device="cuda", generator=gen(5 + n)).to(BF16), torch.randn((n, k), device="cuda", generator=gen(n)).to(BF16)
        rows, s = ops.rms_norm_fp8(b, w["n1"], residual=h)
        got = ops.fp8_forward(rows, *up)
        y, s2 = ops.rms_norm(b, w["n1"], residual=h, out_dtype=F32)
        assert torch.equal(s, s2) and torch.equal(got, ops.fp8_forward(y, *up, out_dtype=BF16))
        y = ops.rms_norm(s, w["n2"])
        losses = ops.linear_cross_entropy(y, w["table"].to(BF16), torch.arange(n, device="cuda"))
        z = y.double() @ w["table"].to(BF16).double().t()
        want = torch.nn.functional.cross_entropy(z, torch.arange(n, device="cuda"), reduction="none")
        assert bool(((losses - want).abs() <= 2e-5 * (1 + want)).all())


def _tiny(seed, width=128):
    from transformers import GPT2Config, GPT2LMHeadModel
    cfg = GPT2Config(n_layer=2, n_embd=width, n_head=4, vocab_size=1000, n_positions=64, bos_token_id=0, eos_token_id=0,
                     resid_pdrop=0.0, embd_pdrop=0.0, attn_pdrop=0.0)
    torch.manual_seed(seed)
    return GPT2LMHeadModel(cfg).cuda().train()


def test_head_backward_matches_the_models_loss():
    """The training loop's head: loss and every gradient are torch's to float32 (products of 128 and 1000 terms through two
    blocks), micro-batches added up."""
    from paper_2608_05088_amd.train import head_backward
    model = _tiny(0)
    plain = copy.deepcopy(model)
    for turn in range(2):
        ids = torch.randint(0, 1000, (3, 40), device="cuda", generator=gen(turn))
        loss = head_backward(model, ids, 0.5)
        want = plain(input_ids=ids, labels=ids).loss
        (want * 0.5).backward()
        assert abs(float(loss) - float(want.detach())) <= 1e-5 * float(want.detach())
    for (n, p), q in zip(model.named_parameters(), plain.parameters()):
        assert float((p.grad - q.grad).norm()) <= 1e-4 * float(q.grad.norm()) + 1e-9, n


@pytest.mark.parametrize("bits", [None, 8, 32])
@pytest.mark.parametrize("rms,fp8", [(False, False), (True, True)])
def test_the_training_loop_runs(bits, rms, fp8):
    from paper_2608_05088_amd.train import head_backward, make_optimizer, use_operators, use_rms_norm
    model = _tiny(1)
    if rms:
        use_rms_norm(model)
    if fp8:
        use_operators(model)
    opt = make_optimizer("malt", model, 1e-3, 1e-3, adamw_bits=bits)
    before = [p.detach().clone() for p in model.parameters()]
    for t in range(3):
        loss = head_backward(model, torch.randint(0, 1000, (2, 32), device="cuda", generator=gen(t)))
        assert bool(loss.isfinite())
        opt.step()
        opt.zero_grad()
    for p, q in zip(model.parameters(), before):
        assert bool(p.isfinite().all()) and not torch.equal(p, q)


def test_adamw_beside_malt_is_torchs(ops):
    """The rest of the model's parameters under the own AdamW in 32 bits and under torch's, three steps: each step's update is
    rounded ten times at most, its size lr, 3 x 10 x 2^-24 of it and the parameter's own roundings."""
    from paper_2608_05088_amd.train import block_matrix, make_optimizer
    a = _tiny(2)
    b = copy.deepcopy(a)
    oa, ob = (make_optimizer("malt", m, 1e-3, 1e-3, adamw_bits=bits) for m, bits in ((a, 32), (b, None)))
    for t in range(3):
        for i, (p, q) in enumerate(zip(a.parameters(), b.parameters())):
            p.grad = torch.randn(p.shape, device="cuda", generator=gen(50 * t + i))
            q.grad = p.grad.clone()
        oa.step(), ob.step()
    for (n, p), q in zip(a.named_parameters(), b.parameters()):
        if block_matrix(n, p):
            assert torch.equal(p, q)
        else:
            assert float((p - q).detach().abs().max()) <= 3 * (40 * 1e-3 * 2.0 ** -24 * 10 + 3 * 2.0 ** -24 * float(q.detach().abs().max())), n


@pytest.mark.parametrize("op", ["head", "norm"])
def test_a_captured_backward_pass_and_an_eager_graph(ops, op):
    """Beside an eager graph of the same leaves on the default stream a captured backward pass is refused, before
    the engine reaches that graph; without one, or with one of another stream, it is captured."""
    x = torch.randn((40, 64), device="cuda", generator=gen(90))
    w = torch.rand((64,) if op == "norm" else (100, 64), device="cuda", generator=gen(91)).requires_grad_()
    y = torch.arange(40, device="cuda")
    dy = torch.randn((40, 64) if op == "norm" else (40,), device="cuda", generator=gen(92))

    def forward():
        return ops.rms_norm(x, w) if op == "norm" else ops.linear_cross_entropy(x, w, y)

    def capture():
        g = torch.cuda.CUDAGraph()
        w.grad = None
        with torch.cuda.graph(g):
            forward().backward(dy)
        return g

    eager = forward()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="default stream"):
        capture()
    torch.cuda.synchronize()
    w.grad = None
    eager.backward(dy)
    want = w.grad.clone()
    del eager
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        held = forward()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for _ in range(2):   # beside a graph of another stream, then beside none
        g = capture()
        for _ in range(3):
            w.grad.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(w.grad, want)
        held = None


@pytest.mark.parametrize("stream", [False, True])
def test_host_tensors_and_no_tensors_are_refused(ops, stream):
    """Before anything is recorded on a stream."""
    kw = dict(stream=torch.cuda.Stream()) if stream else {}
    x, w, y = torch.ones((4, 64), device="cuda"), torch.ones((9, 64), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    gain, st = torch.ones(64, device="cuda"), ops.adamw_state(x)
    torch.cuda.synchronize()
    calls = {
        "loss": (lambda a, b, c: ops.linear_cross_entropy(a, b, c, **kw), (x, w, y)),
        "step": (lambda a, b, c, g, o: ops.linear_cross_entropy_step(a, b, c, grad=g, out=o, **kw),
                 (x, w, y, torch.ones(4, device="cuda"), torch.zeros_like(w))),
        "norm": (lambda a, b, r: ops.rms_norm(a, b, residual=r, **kw), (x, gain, x.clone())),
        "norm_fp8": (lambda a, b, r: ops.rms_norm_fp8(a, b, residual=r, **kw), (x, gain, x.clone())),
        "adamw": (lambda p, g, s, c: ops.adamw_step([p], [g], [s], lr=0.0, step=1, grad_scale=c, **kw),
                  (x.clone(), x, st, torch.ones((), device="cuda"))),
        "moments": (lambda p, s: ops.adamw_moments([p], [s], **kw), (x, st)),
    }
    for name, (call, args) in calls.items():
        call(*args)
        for i, t in enumerate(args):
            with pytest.raises(ValueError):
                call(*args[:i], t.cpu(), *args[i + 1:])
            with pytest.raises((TypeError, ValueError)):
                call(*args[:i], object(), *args[i + 1:])
    with pytest.raises(ValueError):
        ops.adamw_step([], [x], [st], lr=0.0, step=1, **kw)
    with pytest.raises(ValueError):
        ops.adamw_moments([], [st], **kw)
    with pytest.raises(ValueError):
        ops.adamw_step([x], [], [st], lr=0.0, step=1, **kw)
    torch.cuda.synchronize()
