"""What an 8-bit layer keeps for its backward pass, and what that pass refuses (no GPU
needed: refused calls follow no pointer)."""
import os
from ctypes import byref, c_size_t, c_void_p

import pytest

from paper_2608_05088_amd import libmalt as lm


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lm.LIB_PATH):
        from paper_2608_05088_amd import build
        build.build()
    return lm.lib()


def _kept_bytes(L, m, n, k, transposed, need_dx, need_dw):
    kept, fwd, bwd = c_size_t(0), c_size_t(0), c_size_t(0)
    assert L.malt_block_layer_size(m, n, k, transposed, 0, 0, 0, need_dx, need_dw, byref(kept), byref(fwd), byref(bwd)) == lm.MALT_OK
    return kept.value


def _backward(L, m, n, k, transposed, kept, dx, dw):
    n_dw = n if transposed else k
    far = [c_void_p(i << 40) for i in range(1, 6)]   # far apart, whatever the sizes
    return L.malt_block_layer_backward(far[0], 0, m, n, n, k, transposed, far[1], kept, far[2] if dx else None, 0, k,
                                       far[3] if dw else None, 0, n_dw, 0, far[4], 1 << 38, None)


# The second and third: input and weight gradient alone would keep as many bytes as each other.
@pytest.mark.parametrize("m,n,k", [(40, 200, 256), (16384, 16512, 256), (16384, 16512, 512), (1, 1, 1), (129, 1, 300)])
@pytest.mark.parametrize("transposed", [0, 1])
def test_layer_backward_refuses_what_was_kept_for_other_gradients(L, m, n, k, transposed):
    sizes = {(dx, dw): _kept_bytes(L, m, n, k, transposed, dx, dw) for dx in (0, 1) for dw in (0, 1)}
    assert len(set(sizes.values())) == 4
    for asked in ((1, 0), (0, 1), (1, 1)):
        for kept_for, size in sizes.items():
            if kept_for != asked:
                assert _backward(L, m, n, k, transposed, size, *asked) == lm.MALT_ERR_INVALID_ARG, (asked, kept_for)
                assert lm.last_error()
