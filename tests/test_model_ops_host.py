"""What the Python entries of the head's loss, the norm, AdamW and the training loop around them do on the
host, without a GPU.  The kernels are not reached."""
import copy
import os
from types import SimpleNamespace

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
    return torch.zeros(*shape[:-2], shape[-1], shape[-2], dtype=dtype).transpose(-1, -2)


@pytest.mark.parametrize("entry", ["loss", "step", "norm", "norm_fp8", "adamw", "moments"])
def test_copies_are_made_on_the_stream_of_the_work(ops, monkeypatch, entry):
    x, w, y = _turned(2, 3, 40), _turned(50, 40), _turned(3, 2, dtype=I64).t()
    g = _turned(3, 2).t()
    s = object()
    call, inputs = {
        "loss": (lambda: ops.linear_cross_entropy(x, w, y, stream=s), (x, w, y)),
        "step": (lambda: ops.linear_cross_entropy_step(x, w, y, grad=g, stream=s), (x, w, y, g)),
        "norm": (lambda: ops.rms_norm(x, w[0], residual=x, stream=s), (x, w)),
        "norm_fp8": (lambda: ops.rms_norm_fp8(x, w[0], residual=x, stream=s), (x, w)),
        "adamw": (lambda: ops.adamw_step([w], [w], [x], lr=1.0, step=1, stream=s), (w, x)),
        "moments": (lambda: ops.adamw_moments([w], [x], stream=s), (x,)),
    }[entry]
    copies, seen = _Copies(), []

    def on(device, stream, tensors, work):
        seen.append((list(copies.met), [t.data_ptr() for t in tensors if t is not None]))
        raise _Enqueued

    monkeypatch.setattr(ops, "_on", on)
    with copies, pytest.raises(_Enqueued):
        call()
    early, recorded = seen[0]
    assert early == []
    for t in inputs:
        assert t.data_ptr() in recorded


def test_results_written_in_place_are_known_to_autograd(ops, monkeypatch):
    monkeypatch.setattr(ops, "_on", lambda *a: (None, None, None, None))
    out = torch.zeros(5, 4)
    leaf = out.clone().requires_grad_()
    saved = leaf * 1.0
    product = (saved * saved).sum()
    ops.linear_cross_entropy_step(torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=I64), out=saved.detach())
    with pytest.raises(RuntimeError, match="inplace"):
        product.backward()


def test_forward_mode_is_refused(ops, monkeypatch):
    from torch.autograd import forward_ad
    monkeypatch.setattr(ops, "_on", lambda *a: (None, None, None, None))
    y = torch.zeros(3, dtype=I64)
    for call in (lambda t: ops.linear_cross_entropy(t, torch.zeros(4, 5), y), lambda t: ops.linear_cross_entropy(torch.zeros(2, 5), t, y[:2]),
                 lambda t: ops.rms_norm(t, torch.zeros(5)), lambda t: ops.rms_norm(torch.zeros(2, 3), t),
                 lambda t: ops.rms_norm(torch.zeros(3, 5), torch.zeros(5), residual=t)):
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(torch.zeros(3, 5), torch.ones(3, 5))
            with pytest.raises(ValueError, match="reverse-mode"):
                call(dual)
            call(torch.zeros(3, 5))


def test_a_differentiable_call_takes_no_stream(ops):
    x, w = torch.zeros(3, 4, requires_grad=True), torch.zeros(5, 4)
    with pytest.raises(ValueError, match="stream"):
        ops.linear_cross_entropy(x, w, torch.zeros(3, dtype=I64), stream=object())
    with pytest.raises(ValueError, match="stream"):
        ops.rms_norm(x, w[0], stream=object())


def test_arguments_of_the_head(ops):
    x, w, y = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=I64)
    for kw in (dict(x=torch.zeros(3, 5)), dict(y=y[:2]), dict(w=torch.zeros(5)), dict(out=torch.zeros(5, 5)), dict(out=torch.zeros(4, 5).t()),
               dict(accumulate=True), dict(grad=torch.zeros(2)), dict(x=torch.zeros(())), dict(w=torch.zeros(0, 4))):
        a = dict(x=x, w=w, y=y)
        a.update({k: v for k, v in kw.items() if k in a})
        with pytest.raises(ValueError):
            ops.linear_cross_entropy_step(a["x"], a["w"], a["y"], **{k: v for k, v in kw.items() if k not in a})


def test_arguments_of_8_bit_rows(ops):
    values, scales = torch.zeros(33, 256, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.uint8)
    rows = ops.Fp8Rows(torch.zeros(6, 256, dtype=torch.uint8), torch.zeros(2, 256, dtype=torch.uint8), torch.Size((2, 3, 200)))
    for bad in (rows._replace(values=rows.values[:5]), rows._replace(values=torch.zeros(256, 6, dtype=torch.uint8).t()),
                rows._replace(scales=rows.scales[:1]), rows._replace(scales=torch.zeros(2, 512, dtype=torch.uint8)),
                rows._replace(shape=torch.Size((2, 3, 300))), rows._replace(shape=torch.Size((5, 200))), rows._replace(shape=torch.Size(()))):
        with pytest.raises(ValueError):
            ops.fp8_forward(bad, values, scales)
    with pytest.raises(ValueError, match="out_dtype"):
        ops.fp8_forward(rows, values, scales, out_dtype=torch.float16)


# ----------------------------------------------------------------- optimizer, loop
@pytest.fixture()
def steps(monkeypatch):
    """ops.adamw_step and adamw_state stood in for: the calls are kept."""
    from paper_2608_05088_amd import ops
    calls = []
    monkeypatch.setattr(ops, "adamw_state", lambda p, bits=32: torch.zeros((2, p.numel())) if bits == 32 else
                        torch.zeros(-(-p.numel() // 256) * 520, dtype=torch.uint8))

    def step(params, grads, states, **kw):
        calls.append((list(params), list(states), kw))
        for p, st in zip(params, states):
            p.sub_(kw["lr"])
            st.add_(1)

    monkeypatch.setattr(ops, "adamw_step", step)
    return calls


def test_adamw_groups_counts_and_seeds(steps):
    from paper_2608_05088_amd.optim import AdamW
    ps = [torch.nn.Parameter(torch.zeros(n, dtype=t)) for n, t in ((10, F32), (5000, F32), (4096, torch.bfloat16))]
    opt = AdamW([dict(params=ps[:2]), dict(params=ps[2:], lr=0.5, betas=(0.8, 0.9))], lr=0.25, bits=8, seed=7)
    for t in range(3):
        for p in ps:
            p.grad = torch.ones_like(p)
        if t == 1:
            ps[0].grad = None
        opt.step()
    assert [[p.numel() for p in c[0]] for c in steps] == [[10, 5000], [4096], [5000], [4096], [10], [5000], [4096]]
    assert [c[2]["step"] for c in steps] == [1, 1, 2, 2, 2, 3, 3]
    assert {c[2]["lr"] for c in steps} == {0.25, 0.5} and steps[1][2]["betas"] == (0.8, 0.9)
    seeds = [c[2]["seed"] for c in steps]
    assert len(set(seeds)) == len(seeds) and all(0 <= s < 1 << 64 and s >> 32 == 7 for s in seeds)
    assert [opt.state[p]["moments"].dtype for p in ps] == [F32, torch.uint8, torch.uint8]
    assert opt.step(lambda: torch.tensor(3.0)) == 3.0
    for kw in (dict(bits=16), dict(seed=-1), dict(seed=1 << 32)):
        with pytest.raises(ValueError):
            AdamW(ps, **kw)


def test_adamw_state_keeps_its_types(steps, tmp_path):
    """torch's loading would make moments of the parameter's type."""
    from paper_2608_05088_amd.optim import AdamW
    ps = [torch.nn.Parameter(torch.zeros(n, dtype=torch.bfloat16)) for n in (10, 5000)]
    opt = AdamW(ps, bits=8)
    for p in ps:
        p.grad = torch.ones_like(p)
    opt.step()
    torch.save(opt.state_dict(), tmp_path / "o.pt")
    qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    other = AdamW(qs, bits=32)
    other.load_state_dict(torch.load(tmp_path / "o.pt", weights_only=True))
    for p, q in zip(ps, qs):
        assert other.state[q]["step"] == 1
        a, b = opt.state[p]["moments"], other.state[q]["moments"]
        assert a.dtype == b.dtype and torch.equal(a, b) and a.data_ptr() != b.data_ptr()


def test_malt_hands_the_rest_to_either_adamw():
    from paper_2608_05088_amd.optim import MALT, AdamW
    w, b = torch.zeros(8, 16, requires_grad=True), torch.zeros(16, requires_grad=True)
    assert type(MALT([w, b])._adam) is torch.optim.AdamW
    for bits in (8, 32):
        inner = MALT([w, b], adamw_lr=0.5, adamw_betas=(0.8, 0.9), adamw_weight_decay=0.3, adamw_bits=bits)._adam
        assert type(inner) is AdamW and inner.bits == bits
        assert inner.param_groups[0]["lr"] == 0.5 and inner.param_groups[0]["betas"] == (0.8, 0.9)
        assert inner.param_groups[0]["weight_decay"] == 0.3
    assert MALT([w], adamw_bits=8)._adam is None
    with pytest.raises(ValueError, match="adamw_bits"):
        MALT([w, b], adamw_bits=4)


def _model():
    from transformers import GPT2Config, GPT2LMHeadModel
    torch.manual_seed(0)
    return GPT2LMHeadModel(GPT2Config(n_layer=2, n_embd=64, n_head=4, vocab_size=100, n_positions=32, bos_token_id=0,
                                      eos_token_id=0, resid_pdrop=0.0, embd_pdrop=0.0, attn_pdrop=0.0)).train()


def _plain_step(x, w, y, grad=1.0, out=None, accumulate=False):
    x, w = x.detach().requires_grad_(), w.detach().requires_grad_()
    losses = torch.nn.functional.cross_entropy((x @ w.t()).flatten(0, -2), y.flatten(), reduction="none", ignore_index=-100)
    dx, dw = torch.autograd.grad(losses.sum() * grad, (x, w))
    return losses.detach().view(y.shape), dx, out.add_(dw) if accumulate else dw


def test_head_backward_is_the_models_own_loss(monkeypatch):
    from paper_2608_05088_amd import ops
    from paper_2608_05088_amd.train import head_backward
    monkeypatch.setattr(ops, "linear_cross_entropy_step", _plain_step)
    model = _model()
    plain = copy.deepcopy(model)
    for turn in range(2):   # the second micro-batch adds to the first's gradients
        ids = torch.randint(0, 100, (3, 20), generator=torch.Generator().manual_seed(turn))
        loss = head_backward(model, ids, 0.5)
        want = plain(input_ids=ids, labels=ids).loss
        (want * 0.5).backward()
        assert torch.allclose(loss, want.detach(), rtol=1e-5)
        for (n, p), q in zip(model.named_parameters(), plain.parameters()):
            assert torch.allclose(p.grad, q.grad, rtol=1e-4, atol=1e-6), n
    one = head_backward(model, torch.zeros((2, 1), dtype=I64))
    assert float(one) == 0.0


def test_rms_norms_in_the_layer_norms_places(monkeypatch):
    from paper_2608_05088_amd import ops
    from paper_2608_05088_amd.train import use_rms_norm
    seen = []
    monkeypatch.setattr(ops, "rms_norm", lambda x, w, eps: seen.append(w) or x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w)
    model = _model()
    use_rms_norm(model)
    other = copy.deepcopy(model)
    for m in (model, other):
        seen.clear()
        m(input_ids=torch.arange(6)[None]).logits.sum().backward()
        assert len(seen) == 5 and all(any(w is p for p in m.parameters()) for w in seen)
    assert not [n for n, _ in model.named_parameters() if "ln_" in n and n.endswith("bias")]


def test_command_line():
    from paper_2608_05088_amd import train
    with pytest.raises(SystemExit):
        train.main(["--head", "--teacher", "gpt2-small"])
    with pytest.raises(SystemExit):
        train.main(["--adamw-bits", "4"])
