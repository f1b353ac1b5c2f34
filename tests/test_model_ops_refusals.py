"""What the head's loss, AdamW, the norm and the layer on 8-bit rows refuse, on the host, before
any device work (no GPU needed: the pointers are never followed)."""
import ctypes
from ctypes import byref, c_int64, c_size_t, c_void_p

import pytest
import torch

from paper_2608_05088_amd import libmalt as lm

P = [0x1000000000 * i for i in range(1, 12)]   # far apart, aligned
BAD, SHAPE, ALIGN, ALIAS = lm.MALT_ERR_INVALID_ARG, lm.MALT_ERR_SHAPE, lm.MALT_ERR_ALIGNMENT, lm.MALT_ERR_ALIAS


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(lm.LIB_PATH) or not os.path.exists(lm.BINDING_PATH):
        from paper_2608_05088_amd import build
        build.build()
    return lm.lib()


# -------------------------------------------------------------------------- head
def _head(**kw):
    a = lm.malt_linear_loss_t(x=P[0], x_type=1, rows=100, inner=64, ldx=64, weight=P[1], weight_type=1, vocab=1000, ldw=64,
                              labels=P[2], label_type=1, label_stride=1, weights=None, weight_stride=0, weight_value=1.0,
                              losses=P[3], stats=None, stats_given=0, dx=P[4], lddx=64, dweight=P[5], dweight_type=1, lddw=64,
                              accumulate=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(weight=None), BAD), (dict(labels=None), BAD), (dict(x_type=2), BAD), (dict(weight_type=-1), BAD),
    (dict(dweight_type=7), BAD), (dict(label_type=2), BAD), (dict(accumulate=2), BAD), (dict(stats_given=2), BAD),
    (dict(stats_given=1), BAD), (dict(stats_given=1, stats=P[6]), BAD), (dict(losses=None, dx=None, dweight=None), BAD),
    (dict(rows=-1), SHAPE), (dict(rows=65537), SHAPE), (dict(inner=0), SHAPE), (dict(inner=65537, ldx=70000, ldw=70000, lddx=70000, lddw=70000), SHAPE),
    (dict(vocab=0), SHAPE), (dict(vocab=(1 << 22) + 1), SHAPE), (dict(vocab=1 << 22, inner=4096, ldx=4096, ldw=4096, lddx=4096, lddw=4096), SHAPE),
    (dict(ldx=63), SHAPE), (dict(ldw=63), SHAPE), (dict(lddx=63), SHAPE),
    (dict(lddw=63), SHAPE), (dict(ldx=1 << 31), SHAPE), (dict(label_stride=-1), SHAPE), (dict(label_stride=1 << 31), SHAPE),
    (dict(weights=P[7], weight_stride=-1), SHAPE), (dict(x=P[0] + 1), ALIGN), (dict(weight=P[1] + 1), ALIGN),
    (dict(labels=P[2] + 4), ALIGN), (dict(losses=P[3] + 2), ALIGN), (dict(weights=P[7] + 2), ALIGN), (dict(stats=P[6] + 8), ALIGN),
    (dict(dx=P[4] + 1), ALIGN), (dict(dweight=P[5] + 1), ALIGN), (dict(losses=P[0]), ALIAS), (dict(dx=P[0]), ALIAS),
    (dict(dx=P[1]), ALIAS), (dict(dweight=P[1]), ALIAS), (dict(dweight=P[4] + 64), ALIAS), (dict(losses=P[2] + 400), ALIAS),
    (dict(stats=P[5]), ALIAS), (dict(weights=P[4], weight_stride=1), ALIAS),
])
def test_head_refuses(L, kw, code):
    size = c_size_t(0)
    assert L.malt_linear_loss_size(byref(_head(**kw)), byref(size)) == code
    assert L.malt_linear_loss(byref(_head(**kw)), c_void_p(P[10]), 1 << 40, None) == code
    assert lm.last_error()


def test_head_workspace(L):
    size = c_size_t(0)
    a = _head()
    assert L.malt_linear_loss_size(byref(a), byref(size)) == lm.MALT_OK and size.value > 0
    assert L.malt_linear_loss(byref(a), None, 0, None) == BAD
    assert L.malt_linear_loss(byref(a), c_void_p(P[10]), size.value - 1, None) == BAD
    assert L.malt_linear_loss(byref(a), c_void_p(P[10] + 16), size.value, None) == ALIGN
    assert L.malt_linear_loss(byref(a), c_void_p(P[0] - 256), size.value, None) == ALIAS
    assert L.malt_linear_loss(byref(a), c_void_p(P[5]), size.value, None) == ALIAS
    assert L.malt_linear_loss(None, c_void_p(P[10]), 1 << 40, None) == BAD
    assert L.malt_linear_loss_size(byref(a), None) == BAD
    # The vocabulary is worked on in pieces: dz both ways stays within 2 x 512 MiB (three planes each in float32).
    big = _head(rows=65536, vocab=100000, inner=64)
    assert L.malt_linear_loss_size(byref(big), byref(size)) == lm.MALT_OK and size.value < (2 << 30)
    # Losses of few rows take their statistics only: 8 bytes for each 16 columns and the labels' logits, in whole 256 bytes.
    few = _head(rows=1, vocab=50257, inner=1280, ldx=1280, ldw=1280, dx=None, dweight=None)
    assert L.malt_linear_loss_size(byref(few), byref(size)) == lm.MALT_OK and size.value <= 8 * 3142 + 512
    none = _head(rows=0, dweight=None)
    assert L.malt_linear_loss(byref(none), c_void_p(P[10]), 1 << 30, None) == lm.MALT_OK


# ------------------------------------------------------------------------- AdamW
def _adam(n=2, hp=None, **kw):
    a = dict(numel=[1000] * n, params=[P[i] for i in range(n)], grads=[P[3 + i] for i in range(n)],
             states=[P[6 + i] for i in range(n)], pt=bytes(n), gt=bytes(n), bits=bytes([8] * n))
    a.update(kw)
    ptr = lambda xs: None if xs is None else (c_void_p * n)(*xs)  # noqa: E731
    t = lm.malt_adamw_tensors_t(n, None if a["numel"] is None else (c_int64 * n)(*a["numel"]), ptr(a["params"]), a["pt"], ptr(a["grads"]),
                                a["gt"], ptr(a["states"]), a["bits"])
    h = lm.malt_adamw_t(1e-3, 0.9, 0.95, 1e-8, 0.1, 1, 1.0, None, 0)
    for k, v in (hp or {}).items():
        setattr(h, k, v)
    return t, h


@pytest.mark.parametrize("kw,code", [
    (dict(numel=None), BAD), (dict(params=None), BAD), (dict(states=None), BAD), (dict(bits=None), BAD), (dict(pt=None), BAD),
    (dict(params=[None, P[1]]), BAD), (dict(grads=[P[3], None]), BAD), (dict(states=[P[6], None]), BAD), (dict(pt=b"\0\2"), BAD),
    (dict(gt=b"\7\0"), BAD), (dict(bits=bytes([8, 16])), BAD), (dict(numel=[-1, 5]), SHAPE), (dict(numel=[5, (1 << 35) + 1]), SHAPE),
    (dict(params=[P[0] + 2, P[1]]), ALIGN), (dict(grads=[P[3] + 1, P[4]]), ALIGN), (dict(states=[P[6] + 1, P[7]]), ALIGN),
    (dict(params=[P[0], P[0]]), ALIAS), (dict(params=[P[0], P[0] + 3996]), ALIAS), (dict(grads=[P[0], P[4]]), ALIAS),
    (dict(states=[P[6], P[6]]), ALIAS), (dict(states=[P[6], P[6] + 2000]), ALIAS), (dict(states=[P[3], P[7]]), ALIAS),
    (dict(hp=dict(grad_scale_at=P[0])), ALIAS), (dict(hp=dict(grad_scale_at=P[9] + 2)), ALIGN),
    (dict(hp=dict(lr=-1.0)), BAD), (dict(hp=dict(lr=float("nan"))), BAD), (dict(hp=dict(lr=float("inf"))), BAD),
    (dict(hp=dict(beta1=1.0)), BAD), (dict(hp=dict(beta2=-0.1)), BAD), (dict(hp=dict(beta1=float("nan"))), BAD),
    (dict(hp=dict(eps=0.0)), BAD), (dict(hp=dict(eps=1e-60)), BAD), (dict(hp=dict(eps=1e-38)), BAD), (dict(hp=dict(weight_decay=-1.0)), BAD),
    (dict(hp=dict(step=0)), BAD), (dict(hp=dict(grad_scale=float("inf"))), BAD),
])
def test_adamw_refuses(L, kw, code):
    t, h = _adam(**kw)
    assert L.malt_adamw_step(byref(t), byref(h), None) == code
    assert lm.last_error()


def test_adamw_sizes_and_nothing_to_do(L):
    size = c_size_t(0)
    assert L.malt_adamw_state_size(1000, 32, byref(size)) == lm.MALT_OK and size.value == 8000
    assert L.malt_adamw_state_size(1000, 8, byref(size)) == lm.MALT_OK and size.value == 4 * 520
    assert L.malt_adamw_state_size(0, 8, byref(size)) == lm.MALT_OK and size.value == 0
    assert L.malt_adamw_state_size(1000, 4, byref(size)) == BAD
    assert L.malt_adamw_state_size(-1, 8, byref(size)) == SHAPE
    assert L.malt_adamw_state_size(1000, 8, None) == BAD
    t, h = _adam()
    assert L.malt_adamw_step(None, byref(h), None) == BAD and L.malt_adamw_step(byref(t), None, None) == BAD
    t.count = -1
    assert L.malt_adamw_step(byref(t), byref(h), None) == BAD
    t, h = _adam(numel=[0, 0], params=[None, None], grads=[None, None], states=[None, None])
    assert L.malt_adamw_step(byref(t), byref(h), None) == lm.MALT_OK
    # Gradients may be read twice, and lie beside each other.
    ptr = (c_void_p * 2)
    args = ((c_int64 * 2)(1000, 1000), ptr(P[0], P[1]))
    assert L.malt_adamw_moments(2, *args, ptr(P[0], P[3]), None) == ALIAS
    assert L.malt_adamw_moments(2, *args, ptr(P[2], P[2] + 4), None) == ALIAS
    assert L.malt_adamw_moments(2, *args, ptr(P[2], P[3] + 2), None) == ALIGN
    assert L.malt_adamw_moments(2, *args, ptr(P[2], None), None) == BAD
    assert L.malt_adamw_moments(-1, *args, ptr(P[2], P[3]), None) == BAD


# -------------------------------------------------------------------------- norm
def _norm(**kw):
    a = lm.malt_rms_norm_t(x=P[0], type=1, rows=10, width=200, ldx=200, residual=P[1], ldr=200, weight=P[2], weight_type=0, eps=1e-6,
                           sum=P[3], lds=200, y=P[4], y_type=1, ldy=200, values=None, scales=None, rstd=P[5])
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(weight=None), BAD), (dict(type=2), BAD), (dict(weight_type=2), BAD), (dict(y_type=3), BAD),
    (dict(sum=None), BAD), (dict(residual=None), BAD), (dict(y=None), BAD), (dict(values=P[6]), BAD), (dict(values=P[6], scales=P[7]), BAD),
    (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(rows=-1), SHAPE), (dict(rows=(1 << 21) + 1), SHAPE), (dict(width=0), SHAPE),
    (dict(width=16385, ldx=20000, ldr=20000, lds=20000, ldy=20000), SHAPE), (dict(ldx=199), SHAPE), (dict(ldr=199), SHAPE),
    (dict(lds=199), SHAPE), (dict(ldy=199), SHAPE), (dict(x=P[0] + 1), ALIGN), (dict(rstd=P[5] + 2), ALIGN),
    (dict(y=None, values=P[6] + 8, scales=P[7]), ALIGN), (dict(y=P[0]), ALIAS), (dict(sum=P[1]), ALIAS), (dict(y=P[3] + 2), ALIAS),
    (dict(rstd=P[2]), ALIAS), (dict(y=None, values=P[6], scales=P[6] + 16), ALIAS),
])
def test_norm_refuses(L, kw, code):
    assert L.malt_rms_norm(byref(_norm(**kw)), None) == code
    assert lm.last_error()


def _norm_grad(**kw):
    a = lm.malt_rms_norm_grad_t(h=P[0], type=1, rows=10, width=200, ldh=200, weight=P[1], weight_type=0, rstd=P[2], dy=P[3], dy_type=1,
                                lddy=200, dsum=P[4], ldds=200, dx=P[5], lddx=200, dweight=P[6])
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(h=None), BAD), (dict(weight=None), BAD), (dict(rstd=None), BAD), (dict(dy=None), BAD), (dict(dx=None, dweight=None), BAD),
    (dict(type=2), BAD), (dict(dy_type=2), BAD), (dict(width=0), SHAPE), (dict(rows=-1), SHAPE), (dict(ldh=1), SHAPE), (dict(lddy=1), SHAPE),
    (dict(ldds=1), SHAPE), (dict(lddx=1), SHAPE), (dict(rstd=P[2] + 1), ALIGN), (dict(dx=P[0]), ALIAS), (dict(dx=P[4]), ALIAS),
    (dict(dweight=P[1]), ALIAS), (dict(dweight=P[5]), ALIAS), (dict(dx=P[8]), ALIAS), (dict(dy=P[8] + 400), ALIAS),
])
def test_norm_gradient_refuses(L, kw, code):
    assert L.malt_rms_norm_grad(byref(_norm_grad(**kw)), c_void_p(P[8]), 1 << 20, None) == code
    assert lm.last_error()


def test_norm_null_workspace_and_no_rows(L):
    size = c_size_t(1)
    assert L.malt_rms_norm_grad_size(10, 200, 1, byref(size)) == lm.MALT_OK and size.value == 3 * 200 * 4
    assert L.malt_rms_norm_grad(byref(_norm_grad()), None, 0, None) == BAD
    assert L.malt_rms_norm_grad(byref(_norm_grad()), c_void_p(P[8]), size.value - 1, None) == BAD
    assert L.malt_rms_norm_grad(byref(_norm_grad()), c_void_p(P[8] + 4), size.value, None) == ALIGN
    assert L.malt_rms_norm_grad_size(10, 200, 0, byref(size)) == lm.MALT_OK and size.value == 0
    assert L.malt_rms_norm_grad_size(10, 200, 1, None) == BAD
    assert L.malt_rms_norm(None, None) == BAD and L.malt_rms_norm_grad(None, None, 0, None) == BAD
    assert L.malt_rms_norm(byref(_norm(rows=0, x=None, residual=None, sum=None, y=None)), None) == lm.MALT_OK


@pytest.mark.parametrize("kw,code", [
    (dict(xv=None), BAD), (dict(xs=None), BAD), (dict(wv=None), BAD), (dict(ws=None), BAD), (dict(m=0), SHAPE), (dict(k=0), SHAPE),
    (dict(n=0), SHAPE), (dict(ot=5), BAD), (dict(ldo=10), SHAPE), (dict(xv=P[0] + 8), ALIGN), (dict(xs=P[1] + 8), ALIGN),
    (dict(wv=P[2] + 8), ALIGN), (dict(out=P[0]), ALIAS), (dict(out=P[1]), ALIAS), (dict(out=P[2]), ALIAS), (dict(out=P[3]), ALIAS),
])
@pytest.mark.parametrize("m", [3, 100])
def test_layer_on_8_bit_rows_refuses(L, kw, code, m):
    a = dict(xv=P[0], xs=P[1], m=m, k=200, wv=P[2], ws=P[3], n=64, out=P[4], ot=0, ldo=64)
    a.update(kw)
    size = c_size_t(0)
    L.malt_block_matmul_size(max(1, a["m"]), 64, 200, 0, byref(size))
    assert L.malt_block_linear_operand(a["xv"], a["xs"], a["m"], a["k"], a["wv"], a["ws"], a["n"], a["out"], a["ot"], a["ldo"],
                                       P[8] if size.value else None, size.value, None) == code


# ------------------------------------------------------------------------ Python
def test_python_refuses(L):
    from paper_2608_05088_amd import ops
    x, w, y = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: ops.linear_cross_entropy(x, w, y), lambda: ops.linear_cross_entropy_step(x, w, y),
                 lambda: ops.rms_norm(x, w[0]), lambda: ops.rms_norm_fp8(x, w[0]), lambda: ops.adamw_state(x),
                 lambda: ops.adamw_step([x], [x], [x], lr=1.0, step=1), lambda: ops.adamw_moments([x], [x])):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: ops.linear_cross_entropy([1.0], w, y), lambda: ops.rms_norm(3, w), lambda: ops.rms_norm(x.numpy(), w),
                 lambda: ops.rms_norm_fp8(None, w), lambda: ops.adamw_step([1], [x], [x], lr=1.0, step=1),
                 lambda: ops.adamw_moments(["p"], [x]), lambda: ops.adamw_state(3)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ops.rms_norm(x.double(), w[0]), lambda: ops.linear_cross_entropy(x.half(), w, y),
                 lambda: ops.adamw_state(x.int()), lambda: ops.adamw_step([x], [x], [x], lr=1.0, step=1, seed=-1),
                 lambda: ops.adamw_step([x], [x], [x], lr=1.0, step=1, seed=1 << 64)):
        with pytest.raises(ValueError):
            call()
    ops.adamw_step([], [], [], lr=1.0, step=1)
    assert ops.adamw_moments([], []) == []


def test_binding_refuses(L):
    """The C++ host side by itself: its checks come before the card is asked for anything."""
    from paper_2608_05088_amd import ops
    h = ops._host()
    x = torch.zeros(3)
    step = lambda p, g, s: h.adamw_step(p, g, s, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, 1.0, None, 0, 0)  # noqa: E731
    with pytest.raises(ValueError, match="as many"):
        step([x], [], [x])
    with pytest.raises(ValueError, match=r"params\[0\] must be on a GPU"):
        step([x], [x], [x])
    with pytest.raises(TypeError, match=r"grads\[0\] must be a tensor"):
        step([x], [None], [x])
    with pytest.raises(TypeError):
        step(3, [x], [x])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        step([x.int()], [x], [x])
    with pytest.raises(ValueError, match="GPU"):
        h.rms_norm(x, x, None, 1e-6, None, False, 0)
    with pytest.raises(TypeError, match="residual"):
        h.rms_norm(x, x, 5, 1e-6, None, False, 0)
    assert step([], [], []) is None and h.adamw_moments([], [], 0) == []
