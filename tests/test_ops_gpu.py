"""The operators around the optimizer step against plain implementations in 64
bits, where they can go wrong: odd sizes, empty and masked rows, strides, long
offsets, repeated ids, other streams, captured graphs.

Tolerances follow from the arithmetic.  u = 2^-24 is float32's unit roundoff,
2^-8 bfloat16's; a sum of n float32 terms is off by at most n u sum|x|.
"""
import ctypes
import math

import pytest
import torch

from paper_2608_05088_amd import libmalt as lm

pytestmark = pytest.mark.gpu
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
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


def rounding(dtype):
    return torch.finfo(dtype).eps / 2


def pitched(x, extra=5):
    """x as a view whose rows lie further apart."""
    big = torch.full((x.shape[0], x.shape[1] + extra), float("nan"), device=x.device, dtype=x.dtype)
    view = big[:, :x.shape[1]]
    view.copy_(x)
    return view


# ================================================================== token table
@pytest.mark.parametrize("table,out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("tokens,width", [(1, 1), (1, 1280), (5, 3), (67, 64), (300, 257), (1000, 769), (9, 2048)])
def test_lookup(ops, table, out, tokens, width):
    v = 97
    w = randn(1, v, width, dtype=table)
    ids = torch.randint(0, v, (tokens,), device="cuda", generator=gen(2))
    ids[::7] = torch.tensor([-1, v, -100, 1 << 40], device="cuda").repeat(tokens)[:ids[::7].numel()]
    got = ops.embedding(ids, w, scale=3.3, out_dtype=out)
    there = (ids >= 0) & (ids < v)
    want = w.double()[ids.clamp(0, v - 1)] * float(torch.tensor(3.3)) * there[:, None]
    assert got.dtype == out and got.shape == (tokens, width)
    assert bool((got[~there] == 0).all())
    assert bool(((got.double() - want).abs() <= (U + rounding(out)) * 1.01 * want.abs()).all())


def test_lookup_shapes_types_and_pitches(ops):
    w = randn(3, 50, 33)
    ids = torch.randint(0, 50, (4, 6), device="cuda", generator=gen(4))
    want = w[ids]
    assert torch.equal(ops.embedding(ids, w), want)
    assert torch.equal(ops.embedding(ids.int(), w), want)
    assert torch.equal(ops.embedding(ids.t().contiguous().t(), w), want)       # ids of another order
    assert torch.equal(ops.embedding(ids, pitched(w)), want)
    assert torch.equal(ops.embedding(ids, w.t().contiguous().t()), want)       # columns not contiguous
    assert ops.embedding(ids[:0], w).shape == (0, 6, 33)
    assert torch.equal(ops.embedding(ids[0, 0], w), w[ids[0, 0]])


def test_lookup_beyond_32_bit_offsets(ops):
    ld = (1 << 31) - 1   # the third row starts past 2^32 elements, 2^33 bytes
    big = torch.empty(2 * ld + 8, device="cuda", dtype=BF16)
    table = big.as_strided((3, 8), (ld, 1))
    rows = randn(5, 3, 8, dtype=BF16)
    table.copy_(rows)
    assert torch.equal(ops.embedding(torch.tensor([2, 0, 1], device="cuda"), table), rows[[2, 0, 1]])


def _ids(kind, tokens, v, seed):
    g = gen(seed)
    if kind == "same":
        return torch.full((tokens,), v // 2, device="cuda")
    if kind == "zipf":
        u = torch.rand(tokens, device="cuda", generator=g, dtype=torch.float64)
        return (torch.exp(u * math.log(v + 1)).long() - 1).clamp(0, v - 1)
    if kind == "none":
        return torch.full((tokens,), -1, device="cuda")
    ids = torch.randint(0, v, (tokens,), device="cuda", generator=g)
    if kind == "holes":
        ids[torch.rand(tokens, device="cuda", generator=g) < 0.3] = -1
        ids[torch.rand(tokens, device="cuda", generator=g) < 0.1] = v
    return ids


def _check_grad(ids, grad, v, scale, got, old=None):
    there = (ids >= 0) & (ids < v)
    at = ids[there].long()
    width = grad.shape[1]
    want = torch.zeros((v, width), dtype=torch.float64, device="cuda")
    want.index_put_((at,), grad[there].double(), accumulate=True)
    size = torch.zeros_like(want).index_put_((at,), grad[there].double().abs(), accumulate=True)
    n = torch.zeros(v, dtype=torch.float64, device="cuda").index_put_((at,), torch.ones_like(at, dtype=torch.float64),
                                                                       accumulate=True)
    s = float(torch.tensor(scale, dtype=F32))
    want, bound = want * s, (n[:, None] + 2) * U * size * s
    if old is not None:
        want = want + old.double()
        bound = bound + 2 * U * (old.double().abs() + size * s)
    bound = bound + rounding(got.dtype) * want.abs() * 1.01
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("tokens", [0, 1, 63, 64, 65, 256, 257, 2048, 8192, 8193, 40000])
@pytest.mark.parametrize("kind", ["uniform", "same", "zipf", "holes", "none"])
def test_table_gradient(ops, tokens, kind):
    v, width = 1001, 70
    ids = _ids(kind, tokens, v, 7)
    grad = randn(8, tokens, width)
    got = ops.embedding_grad(ids, grad, v, scale=2.5)
    _check_grad(ids, grad, v, 2.5, got)
    assert torch.equal(got, ops.embedding_grad(ids.int(), grad, v, scale=2.5))   # the same bits again


@pytest.mark.parametrize("gtype,ttype", [(F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("v,width,tokens", [(1, 1, 300), (3, 5, 9000), (70000, 257, 700), (300, 1030, 12000), (255, 512, 100)])
def test_table_gradient_types_and_sizes(ops, gtype, ttype, v, width, tokens):
    ids, grad = _ids("zipf", tokens, v, 9), randn(10, tokens, width, dtype=gtype)
    _check_grad(ids, grad, v, 1.0, ops.embedding_grad(ids, grad, v, dtype=ttype))


@pytest.mark.parametrize("tokens", [0, 40, 3000, 20000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_table_gradient_accumulates_into_pitched_rows(ops, tokens, dtype):
    v, width = 333, 130
    ids, grad = _ids("zipf", tokens, v, 11), pitched(randn(12, tokens, width, dtype=dtype))
    old = randn(13, v, width, dtype=dtype)
    out = pitched(old)
    ret = ops.embedding_grad(ids, grad, v, scale=0.5, out=out, accumulate=True)
    assert ret is out
    _check_grad(ids, grad, v, 0.5, out, old)
    unmet = torch.ones(v, dtype=torch.bool, device="cuda")
    unmet[ids] = False
    assert torch.equal(out[unmet], old[unmet])
    fresh = ops.embedding_grad(ids, grad, v, scale=0.5, out=out)
    _check_grad(ids, grad, v, 0.5, fresh)


def test_table_gradient_of_many_tokens(ops):
    """More tokens than a chunk of 32 each: sums of sums."""
    v, tokens = 5000, 600000
    ids, grad = _ids("zipf", tokens, v, 14), randn(15, tokens, 12, dtype=BF16)
    _check_grad(ids, grad, v, 1.0, ops.embedding_grad(ids, grad, v, dtype=F32))


def test_lookup_differentiates(ops):
    v, w = 40, 9
    table = randn(16, v, w).requires_grad_()
    ids = _ids("holes", 100, v, 17).view(10, 10)
    c = randn(18, 10, 10, w)
    (ops.embedding(ids, table, scale=1.5) * c).sum().backward()
    _check_grad(ids.view(-1), c.view(-1, w), v, 1.5, table.grad)
    # The output is linear in the table: a difference is exact up to rounding.
    d = randn(19, v, w)
    with torch.no_grad():
        rise = (ops.embedding(ids, table + d, scale=1.5).double() * c).sum() - (ops.embedding(ids, table, scale=1.5).double() * c).sum()
    scale = (table.abs().sum() + d.abs().sum()) * c.abs().max() * 1.5
    assert abs(float(rise - (table.grad.double() * d).sum())) <= 1000 * U * float(scale)
    # A broadcast gradient, and one of another type.
    t2 = table.detach().to(BF16).requires_grad_()
    ops.embedding(ids, t2, out_dtype=F32).sum().backward()
    _check_grad(ids.view(-1), torch.ones(100, w, device="cuda"), v, 1.0, t2.grad)
    with pytest.raises(ValueError, match="stream"):
        ops.embedding(ids, table, stream=torch.cuda.Stream())


# ================================================================= distillation
def _distill64(z, a, ids, labels, tau, alpha, weight):
    """Losses and gradient in 64 bits, row by row from the definition."""
    z = z.double().cpu()
    n, v = z.shape
    losses, grad = torch.zeros(n, dtype=torch.float64), torch.zeros_like(z)
    for r in range(n):
        w = float(weight[r])
        entries = []
        if a is not None:
            entries = [(int(i), float(x)) for i, x in zip(ids[r].cpu(), a[r].double().cpu()) if 0 <= int(i) < v]
            entries = [e for e in entries if e[1] != -math.inf]
        y = int(labels[r]) if labels is not None else -1
        if entries and alpha < 1:
            x = torch.tensor([e[1] for e in entries], dtype=torch.float64) / tau
            p, lp = torch.softmax(x, 0), torch.log_softmax(x, 0)
            lq = torch.log_softmax(z[r] / tau, 0)
            at = torch.tensor([e[0] for e in entries])
            losses[r] += (1 - alpha) * tau ** 2 * torch.where(p > 0, p * (lp - lq[at]), torch.zeros_like(p)).sum()
            g = torch.exp(lq)
            g.index_put_((at,), -p, accumulate=True)
            if w:
                grad[r] += w * (1 - alpha) * tau * g
        if 0 <= y < v and alpha > 0:
            l1 = torch.log_softmax(z[r], 0)
            losses[r] -= alpha * l1[y]
            g = torch.exp(l1)
            g[y] -= 1
            if w:
                grad[r] += w * alpha * g
    return losses, grad


def _check_distill(got, want, z, tau, alpha, weight, dtype):
    """A row's exponents reach E = (max - min) / tau log2(e) in size and are rounded to u E; with sums of fewer
    than 2^18 terms by threads and trees that keeps probabilities within 2^-19 (1 + E / 16) relative, and
    log-probabilities as much absolutely."""
    losses, grad = got
    wl, wg = want
    zz = z.double().cpu()
    top = torch.where(torch.isfinite(zz), zz, torch.zeros_like(zz)).abs().amax(1)
    rel = 2.0 ** -19 * (1 + top * max(1.0, 1.0 / tau) / 16)
    big = (1 - alpha) * tau ** 2 + alpha
    gl, gg = losses.double().cpu(), grad.double().cpu()
    assert torch.equal(torch.isnan(gl), torch.isnan(wl)) and torch.equal(torch.isinf(gl), torch.isinf(wl))
    f = torch.isfinite(wl)
    assert bool(((gl - wl).abs()[f] <= (rel * big * 2 + 4 * U * wl.abs())[f]).all()), (gl - wl).abs()[f].max()
    assert torch.equal(torch.isnan(gg), torch.isnan(wg))
    scale = weight.double().cpu().abs()[:, None] * big
    bound = rel[:, None] * scale * 2 + rounding(dtype) * wg.abs() * 1.01 + 2.0 ** -133
    ok = torch.isnan(wg) | ((gg - wg).abs() <= bound)
    assert bool(ok.all()), (gg - wg).abs()[~ok].max()
    # Small probabilities are right relatively, too (columns nothing was taken off).
    rows = torch.isfinite(wg).all(1)
    pos = (wg > 2.0 ** -100) & rows[:, None]
    assert bool(((gg - wg).abs()[pos] <= ((4 * rel[:, None] + 2 * rounding(dtype)) * wg + bound * (wg > 1e-3 * scale))[pos]).all() or
                bool(((gg - wg).abs()[pos] <= bound[pos]).all()))


def _case(seed, n, v, k, dtype, spread=3.0):
    g = gen(seed)
    z = randn(seed + 1, n, v, scale=spread, dtype=dtype)
    ids = torch.stack([torch.randperm(v, device="cuda", generator=g)[:k] for _ in range(n)]) if k else None
    a = (z.float().gather(1, ids) + randn(seed + 2, n, k)).to(dtype) if k else None
    labels = torch.randint(0, v, (n,), device="cuda", generator=g)
    weight = randn(seed + 3, n)
    return z, a, ids, labels, weight


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v,k", [(1, 1), (2, 1), (7, 3), (8, 8), (63, 5), (1000, 64), (1025, 65), (4097, 130), (8200, 1024),
                                 (15001, 3), (28673, 8), (53257, 64), (110003, 33), (211001, 7)])
def test_distillation_sizes(ops, dtype, v, k):
    z, a, ids, labels, weight = _case(100 + v, 3, v, k, dtype)
    for tau, alpha in ((1.0, 0.0), (2.0, 0.5), (1.5, 0.25)):
        got = ops.distill_step(z, a, ids, labels, tau=tau, alpha=alpha, grad=weight)
        _check_distill(got, _distill64(z, a, ids, labels, tau, alpha, weight), z, tau, alpha, weight, dtype)
        assert torch.equal(ops.distill_loss(z, a, ids, labels, tau=tau, alpha=alpha), got[0])


@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 3.0])
@pytest.mark.parametrize("alpha", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("mixed", [False, True])
def test_distillation_temperatures(ops, tau, alpha, mixed):
    z, a, ids, labels, weight = _case(200, 6, 517, 20, BF16)
    if mixed:   # a teacher in float32 beside a bfloat16 student, narrow ids and labels
        a, ids, labels = a.float() + 0.01, ids.int(), labels.int()
    got = ops.distill_step(z, a, ids, labels, tau=tau, alpha=alpha, grad=weight)
    _check_distill(got, _distill64(z, a, ids, labels, tau, alpha, weight), z, tau, alpha, weight, BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distillation_of_labels_alone_and_of_a_teacher_alone(ops, dtype):
    z, a, ids, labels, weight = _case(210, 5, 300, 9, dtype)
    got = ops.distill_step(z, None, None, labels, alpha=1.0, grad=weight)
    _check_distill(got, _distill64(z, None, None, labels, 1.0, 1.0, weight), z, 1.0, 1.0, weight, dtype)
    got = ops.distill_step(z, a, ids, None, tau=2.0, alpha=0.0, grad=weight)
    _check_distill(got, _distill64(z, a, ids, None, 2.0, 0.0, weight), z, 2.0, 0.0, weight, dtype)
    got = ops.distill_step(z, a[:, :0], ids[:, :0], labels, tau=2.0, alpha=0.4, grad=weight)
    _check_distill(got, _distill64(z, None, None, labels, 2.0, 0.4, weight), z, 2.0, 0.4, weight, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_distillation_rows_that_lack_something(ops, dtype, tau):
    """Ids and labels out of range, masses of zero, masked logits, rows masked out whole."""
    n, v, k = 14, 203, 6
    z, a, ids, labels, weight = _case(220, n, v, k, dtype)
    inf, nan = math.inf, math.nan
    ids[0] = -1                                  # no teacher
    labels[1] = -100                             # no label
    ids[2], labels[2] = v, v                     # neither
    ids[3], labels[3], z[3] = -1, -1, nan        # neither, and nothing to read
    z[4, :100] = -inf                            # half the vocabulary masked, maybe the teacher's ids too
    ids[4], labels[4] = torch.arange(150, 150 + k), 160
    z[5, :] = -inf                               # no finite logit
    z[6, int(ids[6, 0])] = -inf                  # the teacher names a masked column: an infinite loss
    a[7, 2:] = -inf                              # entries without mass
    a[8] = -inf                                  # none has any
    ids[9, 1], ids[9, 3] = ids[9, 0], ids[9, 0]  # an id named three times
    labels[9] = ids[9, 0]                        # and the label too
    weight[10], z[10, 5] = 0.0, nan              # weight 0: no gradient
    z[11] = torch.finfo(dtype).min               # every logit the type's lowest value
    ids[12, 3:], a[12, 3:] = -1, nan             # no entries: their logits are not read
    a[13], ids[13] = -inf, -1
    z[13], labels[13] = -inf, -1                 # an empty row of padding
    got = ops.distill_step(z, a, ids, labels, tau=tau, alpha=0.5, grad=weight)
    want = _distill64(z, a, ids, labels, tau, 0.5, weight)
    for r in (2, 3, 13):
        assert float(got[0][r]) == 0.0 and bool((got[1][r] == 0).all())
    assert bool((got[1][10] == 0).all())
    # Row 5 has no distribution: loss and gradient are not numbers.
    assert math.isnan(float(got[0][5])) and bool(torch.isnan(got[1][5]).all())
    # Row 10's loss holds its NaN.
    assert math.isnan(float(got[0][10]))
    assert math.isinf(float(got[0][6]))
    keep = [r for r in range(n) if r not in (3, 5, 10, 11, 13)]
    sel = lambda x: x[keep]  # noqa: E731
    _check_distill((sel(got[0]), sel(got[1])), (sel(want[0]), sel(want[1])), sel(z), tau, 0.5, sel(weight), dtype)
    # Row 11: equal logits, so q = 1 / v.
    free = [c for c in range(v) if c not in ids[11].tolist() + [int(labels[11])]]
    q = float(weight[11]) * (0.5 * tau + 0.5) / v
    assert bool(((got[1][11][free].double() - q).abs() <= (2.0 ** -18 + rounding(dtype)) * abs(q)).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distillation_pitches_and_places(ops, dtype):
    n, v, k = 9, 1003, 12
    z, a, ids, labels, weight = _case(230, n, v, k, dtype)
    kw = dict(tau=2.0, alpha=0.5)
    losses, grad = ops.distill_step(z, a, ids, labels, grad=weight, **kw)
    # Rows of other alignments are cut into other vectors, so sums may be added in another order: same bound, not same bits.
    want = _distill64(z, a, ids, labels, 2.0, 0.5, weight)
    for extra in (1, 5, 8):
        got = ops.distill_step(pitched(z, extra), pitched(a), pitched(ids.double()).long(), labels, grad=weight, **kw)
        _check_distill(got, want, z, 2.0, 0.5, weight, dtype)
        out = pitched(torch.zeros_like(z), extra)       # rows of other alignments than the logits'
        got = ops.distill_step(z, a, ids, labels, grad=weight, out=out, **kw)
        assert got[1] is out and torch.equal(got[0], losses) and torch.equal(out, grad)
    wide = torch.stack([labels, labels + 1], 1)
    assert torch.equal(ops.distill_step(z, a, ids, wide[:, 0], grad=weight, **kw)[1], grad)
    same = z.clone()
    assert ops.distill_step(same, a, ids, labels, grad=weight, out=same, **kw)[1] is same   # in place
    assert torch.equal(same, grad)
    lead = ops.distill_step(z.view(3, 3, v), a.view(3, 3, k), ids.view(3, 3, k), labels.view(3, 3),
                            grad=weight.view(3, 3), **kw)
    assert torch.equal(lead[0].view(-1), losses) and torch.equal(lead[1].view(n, v), grad)
    one = ops.distill_step(z[4].clone(), a[4], ids[4], labels[4], grad=weight[4], **kw)
    _check_distill((one[0].view(1), one[1].view(1, v)), (want[0][4:5], want[1][4:5]), z[4:5], 2.0, 0.5, weight[4:5], dtype)
    assert ops.distill_step(z[:0], a[:0], ids[:0], labels[:0], **kw)[1].shape == (0, v)
    with pytest.raises(ValueError):
        ops.distill_step(z, a, ids[:, :5], labels, **kw)
    with pytest.raises(ValueError):
        ops.distill_step(z, a, ids, labels[:3], **kw)
    with pytest.raises(ValueError):
        ops.distill_step(z, a, ids, labels, grad=weight[:3], **kw)
    with pytest.raises(ValueError):
        ops.distill_step(z, a, ids, labels, tau=0.0)


@pytest.mark.parametrize("v", [110003, 211001])
def test_distillation_in_place_beyond_the_registers(ops, v):
    for dtype in (F32, BF16):
        z, a, ids, labels, weight = _case(240, 2, v, 5, dtype)
        want = ops.distill_step(z, a, ids, labels, tau=1.5, alpha=0.5, grad=weight)[1]
        assert torch.equal(ops.distill_step(z, a, ids, labels, tau=1.5, alpha=0.5, grad=weight, out=z)[1], want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vectors", [4863, 5057, 6400, 6402, 12353, 16384, 16390, 20480, 20482, 24640, 33792, 33860])
def test_distillation_where_a_row_meets_the_ends_of_what_is_held(ops, dtype, vectors):
    """Rows that end at, just before or just past registers, LDS and the sizes at which the split changes."""
    v = vectors * (16 // (torch.finfo(dtype).bits // 8)) + 3
    z, a, ids, labels, weight = _case(300 + vectors, 3, v, 9, dtype)
    z[1, -1], z[2, v // 2] = 40.0, 40.0     # the maximum in the last column, and in the middle
    for tau, alpha in ((1.0, 0.0), (2.0, 0.5), (1.5, 0.25)):
        got = ops.distill_step(z, a, ids, labels, tau=tau, alpha=alpha, grad=weight)
        _check_distill(got, _distill64(z, a, ids, labels, tau, alpha, weight), z, tau, alpha, weight, dtype)
        assert torch.equal(ops.distill_loss(z, a, ids, labels, tau=tau, alpha=alpha), got[0])


def test_distillation_beyond_32_bit_offsets(ops):
    ld = (1 << 31) - 8
    z, a, ids, labels, weight = _case(250, 3, 500, 7, BF16)
    want = ops.distill_step(z, a, ids, labels, grad=weight, alpha=0.5)
    far = torch.empty(2 * ld + 512, device="cuda", dtype=BF16).as_strided((3, 500), (ld, 1))
    far.copy_(z)
    got = ops.distill_step(far, a, ids, labels, grad=weight, alpha=0.5, out=far)
    assert torch.equal(got[0], want[0]) and torch.equal(far, want[1])


def test_distillation_differentiates(ops):
    """The backward pass against the one-pass gradient, and that against differences of the losses."""
    z, a, ids, labels, weight = _case(260, 4, 12, 4, F32, spread=1.0)
    kw = dict(tau=2.0, alpha=0.5)
    zz = z.clone().requires_grad_()
    (ops.distill_loss(zz, a, ids, labels, **kw) * weight).sum().backward()
    grad = ops.distill_step(z, a, ids, labels, grad=weight, **kw)[1]
    assert torch.equal(zz.grad, grad)
    zz.grad = None
    ops.distill_loss(zz, a, ids, labels, **kw).sum().backward()     # a broadcast gradient
    assert torch.equal(zz.grad, ops.distill_step(z, a, ids, labels, **kw)[1])
    # Central differences, h = 2^-5: h^2 / 6 times a third derivative below 2 tau^-1 big, and losses
    # rounded to 2^-18 over 2 h.
    h = 2.0 ** -5
    for c in range(12):
        d = torch.zeros_like(z)
        d[:, c] = h
        up, down = ops.distill_loss(z + d, a, ids, labels, **kw), ops.distill_loss(z - d, a, ids, labels, **kw)
        diff = (up.double() - down.double()) / (2 * h) * weight.double()
        assert bool(((diff - grad[:, c].double()).abs() <= (h * h + 2.0 ** -12) * weight.double().abs()).all())


# ================================================================= 8-bit layers
def _rounded64(x, rows, cols):
    """The 8-bit form's values in 64 bits: least 2^e >= 2^-127 with max|block| <= 448 2^e, nearest, ties to even."""
    r, k = x.shape
    full = torch.zeros((-(-r // rows) * rows, -(-k // cols) * cols), dtype=torch.float64)
    full[:r, :k] = x.double().cpu()
    b = full.view(full.shape[0] // rows, rows, full.shape[1] // cols, cols)
    top = b.abs().amax(3).amax(1)
    m, e = torch.frexp(torch.where(top > 0, top, torch.full_like(top, 448.0)))
    e = torch.clamp(e - 9 + (m > 0.875), min=-127)
    unit = torch.ldexp(torch.ones_like(top), e)[:, None, :, None]
    v = b / unit
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return (torch.round(v / step) * step * unit).reshape(full.shape)[:r, :k], e


def _check_product(got, a, b):
    """a b^T of 64-bit operands.  bfloat16 results: products of 8 values are added with 14 bits below the largest
    of them (8 products off by 2^-14 each at most), results rounded to bfloat16.  float32 results: sums in 32 bits,
    whatever their order, of k terms."""
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    diff = (got.double().cpu() - want).abs()
    if got.dtype == BF16:
        assert bool((diff <= 2.0 ** -11 * size + rounding(BF16) * want.abs() * 1.01 + 1e-38).all()), float(diff.max())
    else:
        assert bool((diff <= (a.shape[1] + 2) * U * size + 1e-38).all()), float(diff.max())


def _uneven(seed, r, c, dtype):
    """Blocks of very unequal scale, a row and a column of zeros."""
    x = torch.randn((r, c), device="cuda", generator=gen(seed))
    x *= torch.exp(2 * torch.randn((r, 1), device="cuda", generator=gen(seed + 1)))
    x *= torch.exp(torch.randn((1, c), device="cuda", generator=gen(seed + 2)))
    x[r // 2], x[:, c // 3] = 0, 0
    return x.to(dtype)


@pytest.mark.parametrize("r,c", [(1, 1), (3, 130), (128, 128), (129, 257), (300, 77)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weight_conversion_is_the_definition(ops, r, c, dtype):
    w = _uneven(300, r, c, dtype)
    values, scales = ops.fp8_quantize_weight(w)
    want, e = _rounded64(w, 128, 128)
    assert values.shape == (r, -(-c // 128) * 128) and torch.equal(scales.cpu().int(), e.int() + 127)
    unit = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e).repeat_interleave(128, 0).repeat_interleave(128, 1)
    assert torch.equal(values.double().cpu()[:, :c] * unit[:r, :c], want)
    assert bool((values.float()[:, c:] == 0).all())


def test_conversion_at_the_edges(ops):
    """Largest magnitudes at and just past 448 times a power of two, subnormals, ties, signed zeros."""
    w = torch.zeros(8 * 128, 128, device="cuda")
    tops = [448.0, math.nextafter(448.0, 500), 447.0, 2.0 ** -149, 2.0 ** -126, 3.0e38, 1.0, 0.0]
    for i, t in enumerate(tops):
        w[128 * i, 0] = t
        w[128 * i + 1, :120] = torch.linspace(-1, 1, 120, device="cuda") * t
    values, scales = ops.fp8_quantize_weight(w)
    want, e = _rounded64(w, 128, 128)
    assert torch.equal(scales.cpu().int(), e.int() + 127)
    unit = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e).repeat_interleave(128, 0).repeat_interleave(128, 1)
    assert torch.equal(values.double().cpu() * unit, want)


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 32, 33, 64, 129, 300])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (31, 127), (129, 129), (130, 1000), (1000, 260), (7000, 64)])
def test_layer_on_kept_weights(ops, m, n, k):
    x, w = _uneven(310, m, k, F32), _uneven(320, n, k, F32)
    values, scales = ops.fp8_quantize_weight(w)
    xq, wq = _rounded64(x, 1, 128)[0], _rounded64(w, 128, 128)[0]
    for out in (F32, BF16):
        _check_product(ops.fp8_forward(x, values, scales, out_dtype=out), xq, wq)
    xb = x.to(BF16)
    _check_product(ops.fp8_forward(xb, values, scales), _rounded64(xb, 1, 128)[0], wq)


@pytest.mark.parametrize("m,n,k", [(100, 90, 9000), (256, 256, 2048), (513, 770, 300), (3000, 2700, 200), (40, 40, 20000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_tiles_and_parts(ops, m, n, k, dtype):
    """Both tiles, whole and cut along the contraction, forward and backward."""
    x, w = _uneven(330, m, k, dtype).requires_grad_(), _uneven(340, n, k, dtype).requires_grad_()
    dy = _uneven(350, m, n, dtype)
    y = ops.fp8_linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    wq = _rounded64(w.detach(), 128, 128)[0]
    _check_product(y.detach(), _rounded64(x.detach(), 1, 128)[0], wq)
    _check_product(dx, _rounded64(dy, 1, 128)[0], wq.t().contiguous())
    _check_product(dw, _rounded64(dy, 128, 1)[0].t().contiguous(), _rounded64(x.detach(), 128, 1)[0].t().contiguous())
    assert dx.dtype == dtype and dw.dtype == dtype
    again = torch.autograd.grad(ops.fp8_linear(x, w), (x, w), dy)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("tokens,inner,outer", [(1, 1, 1), (1, 300, 20), (5, 128, 128), (130, 17, 259), (257, 640, 129)])
def test_layer_gradients_at_odd_sizes(ops, tokens, inner, outer):
    for xt, wt in ((F32, BF16), (BF16, F32)):
        x, w = _uneven(360, tokens, inner, xt).requires_grad_(), _uneven(370, outer, inner, wt).requires_grad_()
        dy = _uneven(380, tokens, outer, xt)
        dx, dw = torch.autograd.grad(ops.fp8_linear(x, w), (x, w), dy)
        wq = _rounded64(w.detach(), 128, 128)[0]
        _check_product(dx, _rounded64(dy, 1, 128)[0], wq.t().contiguous())
        _check_product(dw, _rounded64(dy, 128, 1)[0].t().contiguous(), _rounded64(x.detach(), 128, 1)[0].t().contiguous())
        # One gradient alone is the same.
        assert torch.equal(torch.autograd.grad(ops.fp8_linear(x, w.detach()), x, dy)[0], dx)
        assert torch.equal(torch.autograd.grad(ops.fp8_linear(x.detach(), w), w, dy)[0], dw)


@pytest.mark.parametrize("tokens,inner,outer", [(3, 130, 20), (200, 257, 300), (1000, 128, 640)])
def test_layer_on_a_transposed_weight(ops, tokens, inner, outer):
    """A weight that lies (inner, outer): the same blocks, so the same numbers."""
    x, w = _uneven(384, tokens, inner, F32).requires_grad_(), _uneven(385, inner, outer, F32).requires_grad_()
    dy = _uneven(386, tokens, outer, F32)
    y = ops.fp8_linear(x, w, transposed=True)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    wq, xd = _rounded64(w.detach(), 128, 128)[0], x.detach()
    _check_product(y.detach(), _rounded64(xd, 1, 128)[0], wq.t().contiguous())
    _check_product(dx, _rounded64(dy, 1, 128)[0], wq)
    _check_product(dw, _rounded64(xd, 128, 1)[0].t().contiguous(), _rounded64(dy, 128, 1)[0].t().contiguous())
    assert torch.equal(ops.fp8_linear(xd, w.detach(), transposed=True), y.detach())
    assert torch.equal(torch.autograd.grad(ops.fp8_linear(x, w.detach(), transposed=True), x, dy)[0], dx)


def test_layer_against_differences(ops):
    """Whole numbers up to 15 with a 16 in every block are exact in 8 bits, and so is a step of 16: differences
    of the layer give its gradients exactly."""
    g = gen(390)
    m, k, n = 4, 130, 129
    x = torch.randint(-7, 8, (m, k), device="cuda", generator=g).float()
    w = torch.randint(-7, 8, (n, k), device="cuda", generator=g).float()
    dy = torch.randint(-7, 8, (m, n), device="cuda", generator=g).float()
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    dx, dw = torch.autograd.grad(ops.fp8_linear(xg, wg), (xg, wg), dy)
    base = (ops.fp8_linear(x, w).double() * dy).sum()
    for i, j in ((0, 0), (3, 129), (2, 64)):
        up = x.clone()
        up[i, j] += 8
        assert float((ops.fp8_linear(up, w).double() * dy).sum() - base) == 8 * float(dx[i, j])
    for i, j in ((0, 0), (128, 129), (50, 127)):
        up = w.clone()
        up[i, j] += 8
        assert float((ops.fp8_linear(x, up).double() * dy).sum() - base) == 8 * float(dw[i, j])


def test_layer_spreads_what_is_no_number(ops):
    x, w = randn(400, 40, 300), randn(401, 70, 300)
    for bad in (math.nan, math.inf, -math.inf):
        for rows in (5, 40):   # the few-rows kernel and the tiles
            xb = x[:rows].clone()
            xb[3, 200] = bad
            for out in (F32, BF16):
                y = ops.fp8_forward(xb, *ops.fp8_quantize_weight(w), out_dtype=out)
                assert bool(torch.isnan(y[3]).all()) and bool(torch.isfinite(y[:3]).all()) and bool(torch.isfinite(y[4:]).all())


def test_layer_shapes_pitches_and_empty_batches(ops):
    x, w = randn(410, 6, 5, 140), randn(411, 33, 140)
    y = ops.fp8_linear(x, w)
    assert y.shape == (6, 5, 33)
    kept = ops.fp8_quantize_weight(w)
    assert torch.equal(ops.fp8_forward(x, *kept), y)
    assert torch.equal(ops.fp8_linear(pitched(x.view(30, 140), 3), pitched(w, 7)).view(6, 5, 33), y)
    assert torch.equal(ops.fp8_linear(x.view(30, 140).t().contiguous().t(), w).view(6, 5, 33), y)
    assert torch.equal(ops.fp8_forward(x[0, 0], *kept), y[0, 0])
    wg, xg = w.clone().requires_grad_(), x[:0].clone().requires_grad_()
    out = ops.fp8_linear(xg, wg)
    assert out.shape == (0, 5, 33)
    out.sum().backward()
    assert wg.grad.shape == w.shape and bool((wg.grad == 0).all()) and xg.grad.shape == (0, 5, 140)
    assert ops.fp8_forward(x[:0], *kept).shape == (0, 5, 33)
    with pytest.raises(ValueError):
        ops.fp8_linear(x, w[:, :139])
    with pytest.raises(ValueError):
        ops.fp8_forward(x, kept[0][:, :128], kept[1])
    with pytest.raises(ValueError):
        ops.fp8_forward(x, kept[0], kept[1].t())


class Operand:
    """x as an operand along its columns, through the C entries."""

    def __init__(self, x):
        v, s = ctypes.c_size_t(0), ctypes.c_size_t(0)
        r, c = x.shape
        lm._check(lm.lib().malt_block_size(r, c, ctypes.byref(v), ctypes.byref(s)))
        self.buf = torch.empty(v.value + s.value, dtype=torch.uint8, device="cuda")
        self.values, self.scales = self.buf.data_ptr(), self.buf.data_ptr() + v.value
        t = lm.MALT_BFLOAT16 if x.dtype == BF16 else lm.MALT_FLOAT32
        lm._check(lm.lib().malt_block_quantize(x.data_ptr(), t, r, c, x.stride(0), self.values, self.scales, None, None,
                                               torch.cuda.current_stream().cuda_stream))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(50, 60, 200), (50, 60, 6000), (2100, 2200, 128)])
def test_product_accumulates(ops, dtype, m, n, k):
    """The C entry's accumulation, whole and cut along k, into rows of a larger pitch."""
    a, b = randn(420, m, k), randn(421, n, k)
    s = torch.cuda.current_stream().cuda_stream
    qa, qb = Operand(a), Operand(b)
    t = lm.MALT_BFLOAT16 if dtype == BF16 else lm.MALT_FLOAT32
    need = ctypes.c_size_t(0)
    lm._check(lm.lib().malt_block_matmul_size(m, n, k, t, ctypes.byref(need)))
    size = need.value
    assert (size > 0) == (k == 6000)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    old = randn(422, m, n, dtype=dtype)
    out = pitched(old, 3)
    lm._check(lm.lib().malt_block_matmul(m, n, k, qa.values, qa.scales, qb.values, qb.scales, 0, 0, 0, out.data_ptr(), t,
                                         n + 3, 1, ws.data_ptr() if size else None, size, s))
    aq, bq = _rounded64(a, 1, 128)[0], _rounded64(b, 1, 128)[0]
    want, tall = aq @ bq.t() + old.double().cpu(), aq.abs() @ bq.abs().t() + old.double().cpu().abs()
    tol = 2.0 ** -11 * tall + rounding(BF16) * want.abs() * 1.01 if dtype == BF16 else (k + 3) * U * tall
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
    assert bool(torch.isnan(out.as_strided((m - 1, 3), (n + 3, 1), n)).all())   # nothing written between the rows


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [40, 5000])
def test_layer_accumulates_its_weight_gradient(ops, dtype, m):
    n, k = 70, 200
    x, w, dy = _uneven(440, m, k, F32), _uneven(441, n, k, F32), _uneven(442, m, n, F32)
    t = lm.MALT_BFLOAT16 if dtype == BF16 else lm.MALT_FLOAT32
    s = torch.cuda.current_stream().cuda_stream
    kept_n, fwd_n, bwd_n = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_size_t(0)
    lm._check(lm.lib().malt_block_layer_size(m, n, k, 0, 0, 0, t, 0, 1, *map(ctypes.byref, (kept_n, fwd_n, bwd_n))))
    kept, fwd, bwd = (torch.empty(c.value, dtype=torch.uint8, device="cuda") for c in (kept_n, fwd_n, bwd_n))
    y, old = torch.empty((m, n), device="cuda"), randn(443, n, k, dtype=dtype)
    dw = pitched(old, 3)
    lm._check(lm.lib().malt_block_layer_forward(x.data_ptr(), 0, m, k, k, w.data_ptr(), 0, n, k, 0, y.data_ptr(), 0, n, 0, 1,
                                                kept.data_ptr(), kept_n.value, fwd.data_ptr(), fwd_n.value, s))
    lm._check(lm.lib().malt_block_layer_backward(dy.data_ptr(), 0, m, n, n, k, 0, kept.data_ptr(), kept_n.value, None, 0, k,
                                                 dw.data_ptr(), t, k + 3, 1, bwd.data_ptr(), bwd_n.value, s))
    a, b = _rounded64(dy, 128, 1)[0].t().contiguous(), _rounded64(x, 128, 1)[0].t().contiguous()
    want, tall = a @ b.t() + old.double().cpu(), a.abs() @ b.abs().t() + old.double().cpu().abs()
    tol = 2.0 ** -11 * tall + rounding(BF16) * want.abs() * 1.01 if dtype == BF16 else (m + 3) * U * tall
    assert bool(((dw.double().cpu() - want).abs() <= tol).all())


def test_product_beyond_32_bit_offsets(ops):
    """An output whose rows start past 2^32 elements."""
    m, n, k = 3, 40, 130
    a, b = randn(430, m, k), randn(431, n, k)
    s = torch.cuda.current_stream().cuda_stream
    qa, qb = Operand(a), Operand(b)
    ld = (1 << 31) - 1
    out = torch.empty(2 * ld + 64, dtype=BF16, device="cuda").as_strided((m, n), (ld, 1))
    lm._check(lm.lib().malt_block_matmul(m, n, k, qa.values, qa.scales, qb.values, qb.scales, 0, 0, 0, out.data_ptr(),
                                         lm.MALT_BFLOAT16, ld, 0, None, 0, s))
    _check_product(out, _rounded64(a, 1, 128)[0], _rounded64(b, 1, 128)[0])


# ============================================================ streams and graphs
def test_other_streams(ops):
    """On a stream given or current, with inputs made there, results are those of the default stream."""
    z, a, ids, labels, weight = _case(500, 20, 3001, 8, BF16)
    toks, table = _ids("zipf", 3000, 500, 501), randn(502, 500, 96)
    x, w = randn(503, 50, 300), randn(504, 90, 300)
    kept = ops.fp8_quantize_weight(w)
    want = (ops.embedding(toks, table), ops.embedding_grad(toks, randn(505, 3000, 96), 500),
            *ops.distill_step(z, a, ids, labels, alpha=0.5), ops.fp8_forward(x, *kept), ops.fp8_linear(x, w))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for explicit in (True, False):
        kw = dict(stream=side) if explicit else {}
        with (torch.cuda.stream(torch.cuda.current_stream()) if explicit else torch.cuda.stream(side)):
            grad = randn(505, 3000, 96)
            if explicit:
                side.wait_stream(torch.cuda.current_stream())
            got = (ops.embedding(toks, table, **kw), ops.embedding_grad(toks, grad, 500, **kw),
                   *ops.distill_step(z, a, ids, labels, alpha=0.5, **kw), ops.fp8_forward(x, *kept, **kw),
                   ops.fp8_linear(x, w, **kw))
        side.synchronize()
        for p, q in zip(got, want):
            assert torch.equal(p, q)


@pytest.mark.parametrize("tokens", [100, 5000, 20000])
def test_graphs(ops, tokens):
    """Captured once, replayed on changing inputs with other work between: every replay is the eager result."""
    v, w, n = 700, 64, 60
    ids, grad, table = _ids("zipf", tokens, v, 510), randn(511, tokens, w), randn(512, v, w)
    z, a, top, labels, weight = _case(513, n, 2000, 10, F32)
    x, wt, dy = randn(514, n, 300), randn(515, 5000, 300), randn(516, n, 5000)
    x.requires_grad_()
    wt.requires_grad_()

    def run():
        y = ops.fp8_linear(x, wt)
        return (ops.embedding(ids, table), ops.embedding_grad(ids, grad, v),
                *ops.distill_step(z, a, top, labels, tau=2.0, alpha=0.5, grad=weight), y.detach(),
                *torch.autograd.grad(y, (x, wt), dy))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run()
    for i in range(4):
        with torch.no_grad():
            ids.copy_(_ids("zipf", tokens, v, 520 + i))
            for t, s in ((grad, 530), (table, 540), (z, 550), (x, 560), (wt, 570), (dy, 580)):
                t.copy_(randn(s + i, *t.shape))
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(got, want):
            assert torch.equal(p, q), i
