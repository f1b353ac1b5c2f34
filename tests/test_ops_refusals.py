"""What the operators around the optimizer step refuse, on the host, before any
device work (no GPU needed: the pointers are never followed)."""
import ctypes
from ctypes import byref, c_size_t, c_void_p

import pytest

from paper_2608_05088_amd import libmalt as lm

A, B, C, D, E = (c_void_p(0x100000000 * i) for i in range(1, 6))   # far apart, aligned
ODD = c_void_p(0x100000001)


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(lm.LIB_PATH):
        from paper_2608_05088_amd import build
        build.build()
    return lm.lib()


def _lookup(L, **kw):
    a = dict(ids=A, it=1, tokens=4, table=B, tt=0, vocab=10, width=8, ld=8, scale=1.0, out=C, ot=0, old=8)
    a.update(kw)
    return L.malt_embed_lookup(a["ids"], a["it"], a["tokens"], a["table"], a["tt"], a["vocab"], a["width"], a["ld"],
                               a["scale"], a["out"], a["ot"], a["old"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(ids=None), lm.MALT_ERR_INVALID_ARG), (dict(table=None), lm.MALT_ERR_INVALID_ARG),
    (dict(out=None), lm.MALT_ERR_INVALID_ARG), (dict(it=2), lm.MALT_ERR_INVALID_ARG),
    (dict(tt=5), lm.MALT_ERR_INVALID_ARG), (dict(ot=-1), lm.MALT_ERR_INVALID_ARG),
    (dict(tokens=-1), lm.MALT_ERR_SHAPE), (dict(tokens=(1 << 25) + 1), lm.MALT_ERR_SHAPE),
    (dict(vocab=0), lm.MALT_ERR_SHAPE), (dict(width=0), lm.MALT_ERR_SHAPE),
    (dict(width=(1 << 20) + 1, ld=1 << 21, old=1 << 21), lm.MALT_ERR_SHAPE), (dict(ld=7), lm.MALT_ERR_SHAPE),
    (dict(old=7), lm.MALT_ERR_SHAPE), (dict(table=ODD), lm.MALT_ERR_ALIGNMENT), (dict(out=ODD), lm.MALT_ERR_ALIGNMENT),
    (dict(ids=ODD), lm.MALT_ERR_ALIGNMENT), (dict(out=B), lm.MALT_ERR_ALIAS), (dict(out=A), lm.MALT_ERR_ALIAS),
])
def test_lookup_refuses(L, kw, code):
    assert _lookup(L, **kw) == code
    assert lm.last_error()


def test_lookup_of_no_tokens_is_nothing(L):
    assert _lookup(L, tokens=0, ids=None, out=None) == lm.MALT_OK


def _grad(L, **kw):
    a = dict(ids=A, it=1, tokens=1000, grad=B, gt=0, gld=8, scale=1.0, acc=0, d=C, dt=0, vocab=10, width=8, dld=8, ws=D,
             size=1 << 30)
    a.update(kw)
    return L.malt_embed_grad(a["ids"], a["it"], a["tokens"], a["grad"], a["gt"], a["gld"], a["scale"], a["acc"], a["d"],
                             a["dt"], a["vocab"], a["width"], a["dld"], a["ws"], a["size"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(ids=None), lm.MALT_ERR_INVALID_ARG), (dict(grad=None), lm.MALT_ERR_INVALID_ARG),
    (dict(d=None), lm.MALT_ERR_INVALID_ARG), (dict(ws=None), lm.MALT_ERR_INVALID_ARG),
    (dict(size=16), lm.MALT_ERR_INVALID_ARG), (dict(acc=2), lm.MALT_ERR_INVALID_ARG),
    (dict(gt=3), lm.MALT_ERR_INVALID_ARG), (dict(gld=4), lm.MALT_ERR_SHAPE), (dict(dld=4), lm.MALT_ERR_SHAPE),
    (dict(ws=c_void_p(0x400000010)), lm.MALT_ERR_ALIGNMENT), (dict(d=B), lm.MALT_ERR_ALIAS),
    (dict(d=A), lm.MALT_ERR_ALIAS), (dict(ws=C), lm.MALT_ERR_ALIAS), (dict(ws=B), lm.MALT_ERR_ALIAS),
    (dict(vocab=(1 << 25) + 1), lm.MALT_ERR_SHAPE),
])
def test_table_gradient_refuses(L, kw, code):
    assert _grad(L, **kw) == code
    assert lm.last_error()


def test_table_gradient_workspace(L):
    size = c_size_t(1)
    assert L.malt_embed_grad_size(100, 50257, 768, byref(size)) == lm.MALT_OK and size.value == 0
    assert L.malt_embed_grad_size(8192, 50257, 768, byref(size)) == lm.MALT_OK and size.value > 8 * 50257
    assert L.malt_embed_grad_size(8192, 0, 768, byref(size)) == lm.MALT_ERR_SHAPE
    assert L.malt_embed_grad_size(8192, 5, 768, None) == lm.MALT_ERR_INVALID_ARG


def _distill(L, **kw):
    a = lm.malt_distill_t(A.value, 0, 4, 100, 100, B.value, 0, C.value, 1, 3, 3, 3, None, 1, 1, 1.0, 0.5, None, 0, 1.0,
                          D.value, E.value, 100)
    for k, v in kw.items():
        setattr(a, k, v.value if isinstance(v, c_void_p) else v)
    return L.malt_distill(byref(a), None)


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), lm.MALT_ERR_INVALID_ARG), (dict(top=None), lm.MALT_ERR_INVALID_ARG),
    (dict(top_ids=None), lm.MALT_ERR_INVALID_ARG), (dict(losses=None, dlogits=None), lm.MALT_ERR_INVALID_ARG),
    (dict(dtype=2), lm.MALT_ERR_INVALID_ARG), (dict(top_type=2), lm.MALT_ERR_INVALID_ARG),
    (dict(id_type=7), lm.MALT_ERR_INVALID_ARG), (dict(labels=0x900000000, label_type=7), lm.MALT_ERR_INVALID_ARG),
    (dict(tau=0.0), lm.MALT_ERR_INVALID_ARG), (dict(tau=-1.0), lm.MALT_ERR_INVALID_ARG),
    (dict(tau=float("inf")), lm.MALT_ERR_INVALID_ARG), (dict(tau=float("nan")), lm.MALT_ERR_INVALID_ARG),
    (dict(alpha=-0.1), lm.MALT_ERR_INVALID_ARG), (dict(alpha=1.1), lm.MALT_ERR_INVALID_ARG),
    (dict(alpha=float("nan")), lm.MALT_ERR_INVALID_ARG), (dict(rows=-1), lm.MALT_ERR_SHAPE),
    (dict(rows=(1 << 21) + 1), lm.MALT_ERR_SHAPE), (dict(vocab=0), lm.MALT_ERR_SHAPE), (dict(ld=99), lm.MALT_ERR_SHAPE),
    (dict(dld=99), lm.MALT_ERR_SHAPE), (dict(n_top=1025, top_ld=2000, id_ld=2000), lm.MALT_ERR_SHAPE),
    (dict(n_top=-1), lm.MALT_ERR_SHAPE), (dict(top_ld=2), lm.MALT_ERR_SHAPE), (dict(id_ld=2), lm.MALT_ERR_SHAPE),
    (dict(labels=0x900000000, label_stride=-1), lm.MALT_ERR_SHAPE),
    (dict(weights=0x900000000, weight_stride=-1), lm.MALT_ERR_SHAPE), (dict(logits=ODD), lm.MALT_ERR_ALIGNMENT),
    (dict(losses=ODD), lm.MALT_ERR_ALIGNMENT), (dict(top_ids=c_void_p(0x100000004)), lm.MALT_ERR_ALIGNMENT),
    (dict(losses=A), lm.MALT_ERR_ALIAS), (dict(losses=B), lm.MALT_ERR_ALIAS), (dict(dlogits=C), lm.MALT_ERR_ALIAS),
    (dict(dlogits=0x100000004), lm.MALT_ERR_ALIAS), (dict(dlogits=A, dld=101), lm.MALT_ERR_ALIAS),
    (dict(losses=E), lm.MALT_ERR_ALIAS),
])
def test_distillation_refuses(L, kw, code):
    assert _distill(L, **kw) == code
    assert lm.last_error()


def test_distillation_refuses_null_and_takes_no_rows(L):
    assert L.malt_distill(None, None) == lm.MALT_ERR_INVALID_ARG
    assert _distill(L, rows=0) == lm.MALT_OK


def test_operand_sizes(L):
    v, s = c_size_t(0), c_size_t(0)
    assert L.malt_block_size(300, 129, byref(v), byref(s)) == lm.MALT_OK
    assert (v.value, s.value) == (300 * 256, 2 * 512)
    assert L.malt_block_size(0, 5, byref(v), byref(s)) == lm.MALT_ERR_SHAPE
    assert L.malt_block_size(5, (1 << 22) + 1, byref(v), byref(s)) == lm.MALT_ERR_SHAPE
    assert L.malt_block_size(5, 5, None, byref(s)) == lm.MALT_ERR_INVALID_ARG


def _quant(L, **kw):
    a = dict(x=A, t=0, rows=100, cols=200, ld=200, v=B, s=C, tv=D, ts=E)
    a.update(kw)
    return L.malt_block_quantize(a["x"], a["t"], a["rows"], a["cols"], a["ld"], a["v"], a["s"], a["tv"], a["ts"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), lm.MALT_ERR_INVALID_ARG), (dict(t=4), lm.MALT_ERR_INVALID_ARG),
    (dict(v=None, s=None, tv=None, ts=None), lm.MALT_ERR_INVALID_ARG), (dict(s=None), lm.MALT_ERR_INVALID_ARG),
    (dict(tv=None), lm.MALT_ERR_INVALID_ARG), (dict(rows=0), lm.MALT_ERR_SHAPE), (dict(ld=199), lm.MALT_ERR_SHAPE),
    (dict(v=c_void_p(0x200000008)), lm.MALT_ERR_ALIGNMENT), (dict(v=A), lm.MALT_ERR_ALIAS), (dict(tv=B), lm.MALT_ERR_ALIAS),
])
def test_conversion_refuses(L, kw, code):
    assert _quant(L, **kw) == code
    assert lm.last_error()


def test_weight_conversion_refuses(L):
    assert L.malt_block_quantize_weight(A, 0, 10, 10, 10, B, None, C, None) == lm.MALT_ERR_INVALID_ARG
    assert L.malt_block_quantize_weight(A, 0, 10, 10, 10, None, B, None, None) == lm.MALT_ERR_INVALID_ARG
    assert L.malt_block_quantize_weight(A, 0, 10, 10, 10, B, B, None, None) == lm.MALT_ERR_ALIAS


def _matmul(L, **kw):
    a = dict(m=300, n=200, k=256, av=A, asc=B, bv=C, bs=D, blocks=1, i=2, j=1, out=E, ot=0, ldo=200, acc=0,
             ws=c_void_p(0x900000000), size=1 << 30)
    a.update(kw)
    return L.malt_block_matmul(a["m"], a["n"], a["k"], a["av"], a["asc"], a["bv"], a["bs"], a["blocks"], a["i"], a["j"],
                               a["out"], a["ot"], a["ldo"], a["acc"], a["ws"], a["size"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(av=None), lm.MALT_ERR_INVALID_ARG), (dict(bs=None), lm.MALT_ERR_INVALID_ARG),
    (dict(out=None), lm.MALT_ERR_INVALID_ARG), (dict(blocks=2), lm.MALT_ERR_INVALID_ARG),
    (dict(acc=-1), lm.MALT_ERR_INVALID_ARG), (dict(ot=9), lm.MALT_ERR_INVALID_ARG), (dict(m=0), lm.MALT_ERR_SHAPE),
    (dict(k=(1 << 22) + 1), lm.MALT_ERR_SHAPE), (dict(m=1 << 20, n=1 << 20, ldo=1 << 20), lm.MALT_ERR_SHAPE),
    (dict(ldo=199), lm.MALT_ERR_SHAPE), (dict(i=0), lm.MALT_ERR_SHAPE), (dict(j=-1), lm.MALT_ERR_SHAPE),
    (dict(av=c_void_p(0x100000004)), lm.MALT_ERR_ALIGNMENT),
    (dict(blocks=0, bs=c_void_p(0x400000004)), lm.MALT_ERR_ALIGNMENT), (dict(out=ODD), lm.MALT_ERR_ALIGNMENT),
    (dict(out=A), lm.MALT_ERR_ALIAS), (dict(out=C), lm.MALT_ERR_ALIAS), (dict(out=D), lm.MALT_ERR_ALIAS),
    (dict(k=100000, ws=None, size=0), lm.MALT_ERR_INVALID_ARG), (dict(k=100000, size=16), lm.MALT_ERR_INVALID_ARG),
    (dict(k=100000, ws=c_void_p(0x900000010)), lm.MALT_ERR_ALIGNMENT), (dict(k=100000, ws=E), lm.MALT_ERR_ALIAS),
])
def test_product_refuses(L, kw, code):
    if kw.get("k") == 100000:   # cut along k: it needs a workspace
        size = c_size_t(0)
        assert L.malt_block_matmul_size(300, 200, 100000, 0, byref(size)) == lm.MALT_OK and size.value > 0
        kw = dict(kw, i=782)
    assert _matmul(L, **kw) == code
    assert lm.last_error()


def test_kept_layer_refuses(L):
    def call(x=A, xt=0, m=40, k=256, ld=256, w=B, s=C, n=200, out=D, ot=0, ldo=200, ws=E, size=1 << 30):
        return L.malt_block_linear(x, xt, m, k, ld, w, s, n, out, ot, ldo, ws, size, None)
    size = c_size_t(1)
    assert L.malt_block_linear_size(32, 200, 256, 0, byref(size)) == lm.MALT_OK and size.value == 0
    assert L.malt_block_linear_size(33, 200, 256, 0, byref(size)) == lm.MALT_OK and size.value >= 33 * 256 + 2 * 256
    assert call(x=None) == lm.MALT_ERR_INVALID_ARG
    assert call(w=None) == lm.MALT_ERR_INVALID_ARG
    assert call(ws=None, size=0) == lm.MALT_ERR_INVALID_ARG
    assert call(xt=3) == lm.MALT_ERR_INVALID_ARG
    assert call(ld=255) == lm.MALT_ERR_SHAPE
    assert call(m=0) == lm.MALT_ERR_SHAPE
    assert call(w=c_void_p(0x200000008)) == lm.MALT_ERR_ALIGNMENT
    assert call(out=A) == lm.MALT_ERR_ALIAS
    assert call(out=B) == lm.MALT_ERR_ALIAS
    assert call(ws=D) == lm.MALT_ERR_ALIAS


def test_layer_refuses(L):
    kept, fwd, bwd = c_size_t(0), c_size_t(0), c_size_t(0)
    three = (byref(kept), byref(fwd), byref(bwd))
    assert L.malt_block_layer_size(40, 200, 256, 0, 0, 0, 0, 1, 1, *three) == lm.MALT_OK
    assert kept.value >= 256 * 128 + 256 * 256 and fwd.value >= 40 * 256 + 200 * 256 and bwd.value >= 40 * 256 + 200 * 128
    assert L.malt_block_layer_size(40, 200, 256, 0, 0, 0, 0, 0, 0, *three) == lm.MALT_OK and bwd.value == 0
    assert L.malt_block_layer_size(40, 200, 256, 2, 0, 0, 0, 1, 1, *three) == lm.MALT_ERR_INVALID_ARG
    assert L.malt_block_layer_size(0, 200, 256, 0, 0, 0, 0, 1, 1, *three) == lm.MALT_ERR_SHAPE
    assert L.malt_block_layer_size(40, 200, 256, 0, 3, 0, 0, 1, 1, *three) == lm.MALT_ERR_INVALID_ARG
    assert L.malt_block_layer_size(40, 200, 256, 0, 0, 0, 0, 1, 1, None, *three[1:]) == lm.MALT_ERR_INVALID_ARG
    big = 1 << 30

    def forward(x=A, ld=256, w=B, ldw=256, t=0, y=C, ldy=200, k=D, kb=big, ws=E, wb=big):
        return L.malt_block_layer_forward(x, 0, 40, 256, ld, w, 0, 200, ldw, t, y, 0, ldy, 1, 1, k, kb, ws, wb, None)

    assert forward(x=None) == lm.MALT_ERR_INVALID_ARG
    assert forward(ld=255) == lm.MALT_ERR_SHAPE
    assert forward(ldw=255) == lm.MALT_ERR_SHAPE
    assert forward(t=1, ldw=199) == lm.MALT_ERR_SHAPE
    assert forward(t=3) == lm.MALT_ERR_INVALID_ARG
    assert forward(ldy=199) == lm.MALT_ERR_SHAPE
    assert forward(k=None) == lm.MALT_ERR_INVALID_ARG
    assert forward(kb=100) == lm.MALT_ERR_INVALID_ARG
    assert forward(wb=100) == lm.MALT_ERR_INVALID_ARG
    assert forward(ws=c_void_p(0x500000010)) == lm.MALT_ERR_ALIGNMENT
    assert forward(y=A) == lm.MALT_ERR_ALIAS
    assert forward(k=B) == lm.MALT_ERR_ALIAS
    assert forward(ws=D) == lm.MALT_ERR_ALIAS

    def backward(dy=A, ld=200, k=B, kb=big, dx=C, dw=D, acc=0, ws=E, wb=big):
        return L.malt_block_layer_backward(dy, 0, 40, 200, ld, 256, 0, k, kb, dx, 0, 256, dw, 0, 256, acc, ws, wb, None)

    assert backward(dy=None) == lm.MALT_ERR_INVALID_ARG
    assert backward(dx=None, dw=None) == lm.MALT_ERR_INVALID_ARG
    assert backward(acc=2) == lm.MALT_ERR_INVALID_ARG
    assert backward(ld=10) == lm.MALT_ERR_SHAPE
    assert backward(k=None) == lm.MALT_ERR_INVALID_ARG
    assert backward(kb=64) == lm.MALT_ERR_INVALID_ARG
    assert backward(dx=A) == lm.MALT_ERR_ALIAS
    assert backward(dw=C) == lm.MALT_ERR_ALIAS
    assert backward(ws=B) == lm.MALT_ERR_ALIAS


def test_python_refuses_host_tensors_and_types():
    import torch
    from paper_2608_05088_amd import ops
    ids, w = torch.zeros(3, dtype=torch.int64), torch.zeros(4, 5)
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding(ids, w)
    with pytest.raises(TypeError):
        ops.embedding(ids, [[1.0]])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ops.embedding(ids, w.half())
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding_grad(ids, torch.zeros(3, 5), 4)
    with pytest.raises(ValueError, match="GPU"):
        ops.distill_loss(w, None, None)
    with pytest.raises(ValueError, match="GPU"):
        ops.fp8_linear(torch.zeros(2, 5), w)
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        ops.fp8_forward(torch.zeros(2, 5), w, w)
