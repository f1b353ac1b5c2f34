"""What the head's loss takes as workspace, against what include/libmalt.h says of it (no GPU needed)."""
import itertools
from ctypes import byref, c_size_t

import pytest

from paper_2608_05088_amd import libmalt as lm

P = [0x1000000000000 * i for i in range(1, 12)]   # far apart, aligned
F32, BF16 = lm.MALT_FLOAT32, lm.MALT_BFLOAT16
SHARE = 512 << 20


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(lm.LIB_PATH):
        from paper_2608_05088_amd import build
        build.build()
    return lm.lib()


def size(L, m, v, k, xt, wt, dwt, dx=True, dw=True, ldw=None):
    a = lm.malt_linear_loss_t(x=P[0], x_type=xt, rows=m, inner=k, ldx=k, weight=P[1], weight_type=wt, vocab=v, ldw=ldw or k,
                              labels=P[2], label_type=1, label_stride=1, weights=None, weight_stride=0, weight_value=1.0,
                              losses=P[3], stats=None, stats_given=0, dx=P[4] if dx else None, lddx=k,
                              dweight=P[5] if dw else None, dweight_type=dwt, lddw=k, accumulate=0)
    n = c_size_t(0)
    assert L.malt_linear_loss_size(byref(a), byref(n)) == lm.MALT_OK, lm.last_error()
    return n.value


def up(n, to):
    return -(-n // to) * to


def bound(m, v, k, xt, wt, dwt, dx, dw):
    """The header's terms, sizes rounded up to tiles, and a few KB for scales, records and alignment."""
    rows, cols, wide, words = up(m, 256), up(k, 64), up(k, 256), up(v, 256)
    few, grads, mixed = m <= 32, dx or dw, F32 in (xt, wt)
    n = m * up(v, 16) // (16 if few else 128) * 8 + 4 * (rows + words) * (2 if mixed else 1) + 20 * rows + 65536
    if grads or not few:
        n += rows * cols * (4 if xt == F32 else 2)
        n += words * cols * ((4 if wt == F32 else 2) if mixed or k % 64 else 0)
    if not grads:
        return n
    d = 2 * max(3 if dx and xt == F32 or dw and dwt == F32 else 1, 2 if m * v * k < 1 << 32 else 1)
    n += (dx + dw) * min(rows * words * d + 256 * rows * d, max(SHARE, 256 * rows * d))
    if dx:
        b = {(F32, F32): 6, (BF16, F32): 4}.get((xt, wt), 2)
        n += min(wide * words * b, max(SHARE, wide * 256 * b))
        n += max(128 << 20, m * k * 4)
    if dw:
        n += wide * rows * {(F32, F32): 6, (F32, BF16): 4}.get((xt, dwt), 2) + (128 << 20)
    return n


SIZES = [(1, 50257, 1280), (20, 50257, 768), (33, 1000, 64), (300, 1000, 129), (1001, 50257, 901), (4096, 50257, 768),
         (8192, 50257, 1280), (1024, 131072, 2048), (4096, 131072, 4096), (65536, 8200, 64), (65536, 100000, 512), (5, 1 << 22, 576),
         (50, 4000, 16384), (3999, 8190, 1500), (12000, 50257, 5000), (20000, 16600, 14000)]


@pytest.mark.parametrize("m,v,k", SIZES)
def test_the_workspace_is_what_the_header_says(L, m, v, k):
    for xt, wt, dwt in itertools.product((F32, BF16), repeat=3):
        for dx, dw in ((True, True), (True, False), (False, True), (False, False)):
            n, most = size(L, m, v, k, xt, wt, dwt, dx, dw), bound(m, v, k, xt, wt, dwt, dx, dw)
            assert n <= most, (xt, wt, dwt, dx, dw, n / 1e6, most / 1e6)


def test_ordinary_steps_take_less_than_the_logits_and_their_gradient(L):
    for m, k in ((4096, 768), (8192, 768), (8192, 1280)):
        logits = m * 50257 * 4
        assert size(L, m, 50257, k, BF16, BF16, BF16) < 0.6 * 2 * logits
        assert size(L, m, 50257, k, F32, F32, F32) < 2 * logits
        assert size(L, m, 50257, k, BF16, BF16, BF16, False, False) < 0.03 * logits


def test_no_rows_take_no_copies_of_the_weight(L):
    for xt, wt in itertools.product((F32, BF16), repeat=2):
        for dx, dw in ((True, True), (True, False), (False, True), (False, False)):
            assert size(L, 0, 131072, 4096, xt, wt, wt, dx, dw) <= 4096
