"""The head's loss where its numbers run out: rows in which the label alone has mass, operands of
unlike magnitude, weights of zero beside rows that hold no numbers."""
import math

import pytest
import torch

from paper_2608_05088_amd import libmalt as lm

pytestmark = pytest.mark.gpu
F32, BF16, I64 = torch.float32, torch.bfloat16, torch.int64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lm.lib()


@pytest.fixture(scope="module")
def ops():
    from paper_2608_05088_amd import ops as module
    return module


# ------------------------------------------------------------ the label alone
# Natural logarithms: where 2^z is a subnormal number, where it is zero, far from either.
ALONE = (200.0, 3.0, -3.0, -86.0, -89.0, -100.0, -104.0, -110.0, -200.0, -1e4, -1e20)


def _nothing(ops, x, w, y):
    """Loss and gradients are zeros: with probability 1 for the label d = 0, and a product with zero is zero."""
    losses, dx, dw = ops.linear_cross_entropy_step(x, w, y)
    lx, lw = x.clone().requires_grad_(), w.clone().requires_grad_()
    out = ops.linear_cross_entropy(lx, lw, y)
    for t in (losses, dx, dw, out.detach(), *torch.autograd.grad(out.sum(), (lx, lw))):
        assert bool((t == 0).all()), t.flatten()[:8]


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("m", [11, 300])
def test_a_vocabulary_of_one(ops, m, t):
    z = torch.tensor(ALONE, device="cuda").repeat(28)[:m]
    x = torch.zeros((m, 5), device="cuda")
    x[:, 2] = z
    w = torch.zeros((1, 5), device="cuda")
    w[0, 2] = 1.0
    _nothing(ops, x.to(t), w.to(t), torch.zeros(m, dtype=I64, device="cuda"))


@pytest.mark.parametrize("t,far", [(F32, -2.0 ** 110), (BF16, -2.0 ** 110), (F32, -math.inf)])
@pytest.mark.parametrize("m", [11, 300])
def test_all_other_logits_are_infinite(ops, m, t, far):
    """Logits below -2^100 count as -inf.  (A bfloat16 weight of -inf itself is a factor of dx: 0 times it is no number.)

    Logits of float32 hold a row's values to 2^-39 of its largest: beside -1e20 a 1 is nothing, so in the rows that hold
    these two the other logits are 0 and the label's, -1e20, has no mass.  Up to 32 rows there is no such row with a
    label here.  All else is zero, exactly."""
    z = torch.tensor(ALONE, device="cuda").repeat(28)[:m]
    x = torch.zeros((m, 64), device="cuda")
    x[:, 0], x[:, 1] = 1.0, z
    w = torch.zeros((300, 64), device="cuda")
    w[:, 0] = far
    w[7, 0], w[7, 1] = 0.0, 1.0
    y = torch.full((m,), 7, device="cuda")
    y[::5] = -100
    lost = (z < -2.0 ** 39) & (y == 7) & (t == F32)
    if not bool(lost.any()):
        return _nothing(ops, x.to(t), w.to(t), y)
    n = int(lost.sum())
    big = max(far, -(2.0 - 2.0 ** -7) * 2.0 ** 127)   # an infinity is the largest number there
    want_dx, want_dw = torch.zeros((m, 64), dtype=torch.float64, device="cuda"), torch.zeros((300, 64), dtype=torch.float64, device="cuda")
    want_dx[lost, 0], want_dx[lost, 1] = big, -1.0    # the others' mean, less the label's row
    want_dw[:, 0], want_dw[:, 1] = n / 299, n * -1e20 / 299
    want_dw[7, 0], want_dw[7, 1] = -n, n * 1e20
    # Logits of 22 bits, probabilities and sums of float32: (299 + 300) 2^-24 of themselves and 2^-20 more.
    for got, want in zip(ops.linear_cross_entropy_step(x, w, y), (1e20 * lost.double(), want_dx, want_dw)):
        assert bool(((got.double() - want).abs() <= 2.0 ** -14 * want.abs()).all())


@pytest.mark.parametrize("m", [11, 300])
def test_a_row_without_a_finite_logit_is_no_number(ops, m):
    x = torch.ones((m, 8), device="cuda")
    w = torch.full((40, 8), -2.0 ** 110, device="cuda")
    losses, dx, _ = ops.linear_cross_entropy_step(x, w, torch.zeros(m, dtype=I64, device="cuda"))
    assert bool(losses.isnan().all()) and bool(dx.isnan().all())


# ------------------------------------------------------ operands of unlike magnitude
@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("p", [112, -112])
@pytest.mark.parametrize("m", [20, 300])
def test_large_rows_beside_small_ones(ops, m, p, xt):
    """x 2^-p and weight 2^p have the logits of x and weight, of a size that float32 holds; their scales, taken
    one after the other, would pass its range.  Losses have the same bits: powers of two are exact.
    The gradients are those of x and weight times 2^p and 2^-p.  Of those near 2^-112 the planes, the products and their
    sums may lie below float32's smallest normal number and be taken as zero, off by less than 2^-126 each: for each of n
    terms three planes (times |d| <= 1), six products and six additions, and the result: 16 n 2^-126 at most.  Beside
    that float32's sums are off by n + 8 roundings of the terms' sizes, and three products below 2^-24 are left out."""
    v, k = 257, 65
    g = torch.Generator(device="cuda")
    g.manual_seed(m + p)
    w = torch.randn((v, k), device="cuda", generator=g)
    y = torch.randint(0, v, (m,), device="cuda", generator=g)
    x = (torch.randn((m, k), device="cuda", generator=g) + w[y]).to(xt)
    want = ops.linear_cross_entropy_step(x, w, y)
    got = ops.linear_cross_entropy_step(x * 2.0 ** -p, w * 2.0 ** p, y)
    assert torch.equal(got[0], want[0])
    z = x.double() @ w.double().t()
    d = torch.softmax(z, 1)
    d[torch.arange(m, device="cuda"), y] -= 1.0
    u = 2.0 ** -24
    for i, (a, b, power, n) in enumerate(((d, w, p, v), (d.t(), x, -p, m))):
        one, two = want[1 + i].double(), got[1 + i].double() * 2.0 ** -power
        size = a.abs() @ b.double().abs()
        lost = 16 * n * 2.0 ** (-126 - power)
        tol = 2 * (n + 16) * u * size + lost + (2 * torch.finfo(want[1 + i].dtype).eps / 2 * one.abs() * 1.01) + 1e-38
        assert bool(((two - one).abs() <= tol).all()), (i, float(((two - one).abs() / tol).max()))


# ------------------------------------------------------- the weight turned by pieces
@pytest.mark.parametrize("m,v,k,xt,wt,pitch", [(40, 90000, 1024, F32, F32, 0), (33, 131001, 2000, F32, F32, 0), (300, 140003, 1029, BF16, F32, 3),
                                               (20, 300001, 1000, BF16, BF16, 1)])
def test_large_weights_are_turned_by_pieces(ops, m, v, k, xt, wt, pitch):
    """Where the transposed weight passes its share of memory it is packed again for each piece of the vocabulary: two
    pieces, four with a short last one, two of a pitched weight in two planes; two of one plane."""
    from test_head_gpu import Exact, inputs
    x, w, y = inputs(m + v, m, v, k, xt, wt)
    if pitch:
        big = torch.full((v, k + pitch), float("nan"), device="cuda", dtype=wt)
        big[:, :k] = w
        w = big[:, :k]
    y[0], y[1] = v - 1, 0
    Exact(x, w, y).check(*ops.linear_cross_entropy_step(x, w, y))


# ------------------------------------------------------------------ weights, sums
@pytest.mark.parametrize("zero", [0.0, "device"])
@pytest.mark.parametrize("m", [20, 100])
@pytest.mark.parametrize("t", [F32, BF16])
def test_a_weight_of_zero_leaves_nothing(ops, m, t, zero):
    """One weight for all rows, rows that hold no numbers among them: every gradient is zero."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    x = torch.randn((m, 64), device="cuda", generator=g).to(t)
    w = torch.randn((300, 64), device="cuda", generator=g).to(t)
    y = torch.randint(0, 300, (m,), device="cuda", generator=g)
    x[6] = float("nan")
    losses, dx, dw = ops.linear_cross_entropy_step(x, w, y, grad=torch.zeros((), device="cuda") if zero == "device" else zero)
    assert bool(losses[6].isnan()) and bool(losses[:6].isfinite().all())
    assert bool((dx == 0).all()) and bool((dw == 0).all())


def test_accumulated_gradients_are_one_sum(ops):
    """A float32 gradient is added once to what was there: its rounded sum, bit by bit."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x, w = (torch.randn(s, device="cuda", generator=g).to(BF16) for s in ((300, 128), (700, 128)))
    y = torch.randint(0, 700, (300,), device="cuda", generator=g)
    out = torch.empty((700, 128), device="cuda")
    one = ops.linear_cross_entropy_step(x, w, y, out=out)[2].clone()
    before = torch.randn((700, 128), device="cuda", generator=g) * 1e-3
    out.copy_(before)
    ops.linear_cross_entropy_step(x, w, y, out=out, accumulate=True)
    assert torch.equal(out, before + one)
