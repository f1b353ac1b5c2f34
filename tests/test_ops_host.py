"""What the operators' Python entries do on the host, without a GPU: where copies
are made, what is refused, what autograd is told.  The kernels are not reached."""
import os

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2608_05088_amd import libmalt as lm

F32, I64 = torch.float32, torch.int64


@pytest.fixture()
def ops(monkeypatch):
    """The module with tensors of the host let through its checks."""
    if not os.path.exists(lm.LIB_PATH):
        from paper_2608_05088_amd import build
        build.build()
    from paper_2608_05088_amd import ops as module
    monkeypatch.setattr(module, "_tensor", lambda *a, **k: None)
    return module


class _Copies(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.met = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if func.overloadpacket.__name__ in ("clone", "copy_", "_to_copy", "_reshape_copy"):
            self.met.append(str(func))
        return func(*args, **(kwargs or {}))


class _Enqueued(Exception):
    pass


def _turned(*shape, dtype=F32):
    """A tensor of a shape whose last two dimensions lie the other way round."""
    return torch.zeros(*shape[:-2], shape[-1], shape[-2], dtype=dtype).transpose(-1, -2)


def _strided_calls(ops):
    """Every entry that takes a stream, on inputs that have to be laid out anew, and those inputs."""
    ids, table = _turned(4, 6, dtype=I64), _turned(50, 8)
    grad = _turned(4, 6, 8)
    z, a, top = _turned(2, 3, 90), _turned(2, 3, 5), _turned(2, 3, 5, dtype=I64)
    y, w = _turned(3, 2, dtype=I64).t(), _turned(3, 2).t()
    y, w = y.t().contiguous().t(), w.t().contiguous().t()
    x, weight = _turned(2, 3, 140), _turned(33, 140)
    values, scales = torch.zeros(33, 256, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.uint8)
    s = object()
    return {
        "embedding": (lambda: ops.embedding(ids, table, stream=s), (ids, table)),
        "embedding_grad": (lambda: ops.embedding_grad(ids, grad, 50, stream=s), (ids, grad)),
        "distill_loss": (lambda: ops.distill_loss(z, a, top, y, alpha=0.5, stream=s), (z, a, top, y)),
        "distill_step": (lambda: ops.distill_step(z, a, top, y, alpha=0.5, grad=w, stream=s), (z, a, top, y, w)),
        "fp8_linear": (lambda: ops.fp8_linear(x, weight, stream=s), (x, weight)),
        "fp8_linear transposed": (lambda: ops.fp8_linear(x, weight.t(), transposed=True, stream=s), (x, weight)),
        "fp8_quantize_weight": (lambda: ops.fp8_quantize_weight(weight, stream=s), (weight,)),
        "fp8_forward": (lambda: ops.fp8_forward(x, values, scales, stream=s), (x, values, scales)),
    }


@pytest.mark.parametrize("entry", ["embedding", "embedding_grad", "distill_loss", "distill_step", "fp8_linear",
                                   "fp8_linear transposed", "fp8_quantize_weight", "fp8_forward"])
def test_copies_are_made_on_the_stream_of_the_work(ops, monkeypatch, entry):
    """A layout copy made before the given stream is current is ordered before nothing that runs there."""
    call, inputs = _strided_calls(ops)[entry]
    copies = _Copies()
    seen = []

    def on(device, stream, tensors, work):
        seen.append((list(copies.met), [t.data_ptr() for t in tensors if t is not None]))
        raise _Enqueued

    monkeypatch.setattr(ops, "_on", on)
    with copies, pytest.raises(_Enqueued):
        call()
    early, recorded = seen[0]
    assert early == []
    for t in inputs:      # what the stream reads is not handed out again before it has
        assert t.data_ptr() in recorded


def test_results_written_in_place_are_known_to_autograd(ops, monkeypatch):
    """A tensor given as `out` has a new version, through a detached view as well; one made in inference mode has none."""
    monkeypatch.setattr(ops, "_on", lambda *a: (None, None))
    ids, grad, z = torch.zeros(3, dtype=I64), torch.zeros(3, 5), torch.zeros(3, 7)
    for call, out in ((lambda out: ops.embedding_grad(ids, grad, 4, out=out), torch.zeros(4, 5)),
                      (lambda out: ops.distill_step(z, None, None, ids, out=out), z)):
        leaf = out.clone().requires_grad_()
        saved = leaf * 1.0
        product = (saved * saved).sum()
        call(saved.detach())
        with pytest.raises(RuntimeError, match="inplace"):
            product.backward()
        with torch.inference_mode():
            inner = torch.zeros_like(out)
        call(inner)
    outer = torch.zeros(4, 5)
    with torch.inference_mode():
        ops.embedding_grad(ids, grad, 4, out=torch.zeros(4, 5))
        ops.embedding_grad(ids, grad, 4, out=outer)


def test_forward_mode_is_refused(ops, monkeypatch):
    """A dual tensor has no requires_grad, so nothing else would tell that its tangent is dropped."""
    from torch.autograd import forward_ad
    monkeypatch.setattr(ops, "_on", lambda *a: (None, None))
    ids, labels = torch.zeros(3, dtype=I64), torch.zeros(3, dtype=I64)
    calls = [lambda w: ops.embedding(ids, w), lambda z: ops.distill_loss(z, None, None, labels),
             lambda x: ops.fp8_linear(x, torch.zeros(4, 5)), lambda w: ops.fp8_linear(torch.zeros(2, 5), w),
             lambda w: ops.fp8_linear(torch.zeros(2, 3), w, transposed=True)]
    for call in calls:
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(torch.zeros(3, 5), torch.ones(3, 5))
            assert not dual.requires_grad
            with pytest.raises(ValueError, match="reverse-mode"):
                call(dual)
            call(torch.zeros(3, 5))
        call(torch.zeros(3, 5))
    with pytest.raises(ValueError, match="reverse-mode"):
        torch.func.jvp(calls[0], (torch.zeros(3, 5),), (torch.ones(3, 5),))


def test_rows_too_far_apart_are_copied(ops):
    """The kernels take row pitches below 2^31 elements; the last token of (2, 65536, 50257) logits lies further apart."""
    last = torch.empty((2, 65536, 50257), dtype=torch.bfloat16, device="meta")[:, -1]
    assert last.stride(0) >= 1 << 31
    x, ld = ops._rows(last)
    assert x.is_contiguous() and ld == 50257
    near = torch.empty((2, 1 << 15, 1 << 15), dtype=torch.bfloat16, device="meta")[:, -1]
    x, ld = ops._rows(near)
    assert x is near and ld == 1 << 30
    edge = torch.empty_strided((3, 8), ((1 << 31) - 1, 1), device="meta")
    assert ops._rows(edge)[1] == (1 << 31) - 1
    one = torch.empty_strided((1, 8), (1 << 40, 1), device="meta")
    assert ops._rows(one)[1] == 8
