"""Microscaled contractions at the ends of their formats: groups of zeros and of the least and largest scales, elements and groups that are no
numbers, sums of very many terms.  References in 64 bits; bounds as in test_gpu_mx.py, with what underflows counted apart.
"""
import numpy as np
import pytest

from oracle import mx_ref as mx
from tests.test_gpu_mx import U, _bound, _dev, _mx, _np, _out, _rows

pytestmark = pytest.mark.gpu
FEW = (1, 4, 5, 16)               # rows of a product that a kernel of its own takes; 17 and 300 go by tiles


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.sat_create(0, 0)
    yield c
    B.sat_destroy(c)


def _lost(m, k):
    """What may be lost to underflow: a few rows are rounded to the least fp32 number once a group; tiles may drop a product below the least normal one."""
    return ((k + 31) // 32) * 2.0 ** -149 if m in FEW else k * 2.0 ** -126


# largest element of a group and the 4-bit scale byte that it gets
SIZES = [(0.0, 0), (2.0 ** -128, 0), (6 * 2.0 ** -127, 0), (6 * 2.0 ** -126, 1), (6 * 2.0 ** -20, 107), (5.0, 127), (6 * 2.0 ** 30, 157), (3.4 * 2.0 ** 126, 253)]


def _group(rng, size, signed):
    g = size * rng.uniform(0.1, 1.0, 32)
    g[rng.integers(32)] = size
    return (g * rng.choice([-1.0, 1.0], 32) if signed else g).astype(np.float32)


@pytest.mark.parametrize("m", [1, 4, 5, 16, 17, 300])
@pytest.mark.parametrize("stored", [False, True])
def test_every_pair_of_scales(B, ctx, m, stored):
    """One group to a row, so that a result comes from one pair of scales; all elements positive, so that what is too large has a sign."""
    rng = np.random.default_rng(m)
    w = np.stack([_group(rng, s, False) for s, _ in SIZES for _ in range(3)])
    wq, wv = _mx(B, w, 4)
    for shift in range(0, len(SIZES), m):
        which = [SIZES[(shift + r) % len(SIZES)] for r in range(m)]
        a = np.stack([_group(rng, s, False) for s, _ in which])
        assert [int(b) for b in mx.quantise(a, 4)[1][:, 0]] == [b for _, b in which]
        aq, av = _mx(B, a, 4)
        out = _out(m, len(w))
        B.sat_mx_dense_nt(ctx, aq if stored else _dev(a), wq, None, out)
        B.sat_sync_status(ctx)
        got, want = _np(out), av @ wv.T
        there = want <= np.finfo(np.float32).max
        assert np.all(np.abs(got - want)[there] <= (_bound(av, wv.T, 32) + _lost(m, 32))[there])
        assert not np.isfinite(got[~there]).any()


@pytest.mark.parametrize("m", [1, 4, 5, 16, 17, 300])
@pytest.mark.parametrize("stored", [False, True])
@pytest.mark.parametrize("k", [32, 150])
def test_zero_and_tiny_groups_beside_others(B, ctx, m, stored, k):
    import torch
    rng = np.random.default_rng(100 * m + k)
    n, groups = 70, (k + 31) // 32
    sizes = np.array([0.0, 0.0, 2.0 ** -128, 6 * 2.0 ** -126, 1.0, 3.0])
    make = lambda rows: np.concatenate([np.stack([_group(rng, s, True) for s in rng.choice(sizes, rows)]) for _ in range(groups)], axis=1)[:, :k]
    a, w, bias = make(m), make(n), rng.normal(size=n).astype(np.float32)
    a[0], w[3], w[n - 1] = 0.0, 0.0, 0.0                          # whole rows
    aq, av = _mx(B, a, 4)
    wq, wv = _mx(B, w, 4)
    for b in (None, bias):
        out, want = _out(m, n), av @ wv.T + (0.0 if b is None else b)
        B.sat_mx_dense_nt(ctx, aq if stored else _dev(a), wq, None if b is None else torch.from_numpy(b).cuda(), out)
        B.sat_sync_status(ctx)
        got = _np(out)
        assert np.isfinite(got).all()
        assert np.all(np.abs(got - want) <= _bound(av, wv.T, k) + _lost(m, k) + (0.0 if b is None else U * (np.abs(want) + np.abs(b))))
        empty = np.zeros(n) if b is None else bias.astype(np.float64)
        assert np.array_equal(got[0], empty) and (got[:, 3] == empty[3]).all() and (got[:, n - 1] == empty[n - 1]).all()


@pytest.mark.parametrize("m", [1, 4, 5, 16, 17, 300])
@pytest.mark.parametrize("stored", [False, True])
def test_groups_that_are_no_numbers(B, ctx, m, stored):
    """They reach their row or column of results and nothing else, groups of zeros on the other side included."""
    rng = np.random.default_rng(m)
    k, n = 96, 72
    a, w = _rows(rng, m, k), rng.normal(size=(n, k)).astype(np.float32)
    a[:, 32:64], w[9, 32:64] = 0.0, 0.0
    bad = np.zeros((m, n), dtype=bool)
    if m > 1:
        a[m - 1, 70], a[m // 2, 5] = np.inf, np.nan
        bad[[m - 1, m // 2]] = True
    w[5, 40] = np.nan                                            # its group meets only zeros
    w[71, 3] = -np.inf
    bad[:, [5, 71]] = True
    aq, av = _mx(B, a, 4)
    wq, wv = _mx(B, w, 4)
    out = _out(m, n)
    B.sat_mx_dense_nt(ctx, aq if stored else _dev(a), wq, None, out)
    B.sat_sync_status(ctx)
    got, want = _np(out), av @ wv.T
    assert np.array_equal(np.isnan(got), bad) and np.array_equal(np.isnan(want), bad)
    av, wv = np.nan_to_num(av), np.nan_to_num(wv)
    assert np.all(np.abs(got - want)[~bad] <= (_bound(av, wv.T, k) + _lost(m, k))[~bad])


# ---- e4m3's codes of no number --------------------------------------------------------------------------------------------------
def _planted(B, x, where):
    """The 8-bit codes of x with 0x7F (even columns) or 0xFF at `where`, on the GPU, and what they stand for."""
    import torch
    codes, scales = mx.quantise(x, 8)
    rows, d = x.shape
    c = codes[:, :d]
    c[where] = np.broadcast_to(np.where(np.arange(d) % 2 == 0, 0x7F, 0xFF).astype(np.uint8), c.shape)[where]
    st = torch.zeros((rows, (scales.shape[1] + 3) // 4 * 4), dtype=torch.uint8, device="cuda")
    st[:, :scales.shape[1]] = torch.from_numpy(scales).cuda()
    values = mx.dequantise(codes, scales, d, 8)
    assert np.array_equal(np.isnan(values), where)
    return B.make_mx(torch.from_numpy(codes).cuda(), st, d, B.SAT_MX8), values


@pytest.mark.parametrize("rows,d,others", [(1, 1, 1), (5, 33, 9), (64, 300, 70), (200, 256, 300), (3000, 130, 40)])
@pytest.mark.parametrize("phase", [0, 1, 2])
def test_codes_of_no_number(B, ctx, rows, d, others, phase):
    """Matrices encoded elsewhere may hold them.  They read as NaN wherever they are read and reach their column of the stored matrix only:
    every column, every third one bad, each at another row."""
    import torch
    rng = np.random.default_rng(rows + d + phase)
    x = rng.normal(size=(rows, d)).astype(np.float32) * 300
    where = np.zeros((rows, d), dtype=bool)
    cols = np.arange(phase % d, d, 3)
    where[(7 * cols) % rows, cols] = True
    q, values = _planted(B, x, where)
    back = _out(rows, d)
    B.sat_mx_dequantise(ctx, q, back)
    assert np.array_equal(_np(back), values, equal_nan=True)
    bad, clean = where.any(0), np.nan_to_num(values)
    a = rng.normal(size=(others, rows)).astype(np.float32)
    a[0] = 0.0                                                   # nothing times no number is no number
    out = _out(others, d)
    B.sat_mx_dense_nn(ctx, _dev(a), q, out)
    got = _np(out)
    assert np.array_equal(np.isnan(got), np.broadcast_to(bad, got.shape))
    a = a.astype(np.float64)
    assert np.all(np.abs(got - a @ clean)[:, ~bad] <= _bound(a, clean, rows)[:, ~bad] + 1e-44)
    g = rng.normal(size=(rows, others)).astype(np.float32)
    g[:, others - 1] = 0.0
    gw, gb = torch.zeros((d, others), device="cuda"), torch.zeros(others, device="cuda")
    B.sat_mx_dense_tn(ctx, q, _dev(g), gw, gb)
    B.sat_sync_status(ctx)
    got = _np(gw)
    assert np.array_equal(np.isnan(got), np.broadcast_to(bad[:, None], got.shape)) and np.isfinite(_np(gb)).all()
    g = g.astype(np.float64)
    assert np.all(np.abs(got - clean.T @ g)[~bad] <= _bound(clean.T, g, rows)[~bad] + 1e-44)


# ---- very long sums ----------------------------------------------------------------------------------------------------------------
LONG, LONG_D, LONG_N = 1_000_000, 4609, 1793                     # 152 tiles: a pair of SMs has more than one each, so the terms are not split


@pytest.fixture(scope="module")
def long_gradient(B, ctx):
    """Weight and bias gradient of a million rows.  Codes: 0.5 to 1.875, scales one; gradients 2^j (1 + 2^-7 - 2^-12), whose second bf16 term is as
    large as it can be, the last column a third throughout."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    groups = (LONG_D + 31) // 32
    codes = torch.randint(0x30, 0x40, (LONG, 32 * groups), dtype=torch.uint8, device="cuda", generator=gen)
    codes[:, LONG_D:] = 0
    q = B.make_mx(codes, torch.full((LONG, (groups + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda"), LONG_D, B.SAT_MX8)
    g = torch.zeros((LONG, (LONG_N + 3) // 4 * 4), device="cuda")[:, :LONG_N]
    g.copy_(torch.randint(0, 3, (LONG, LONG_N), dtype=torch.uint8, device="cuda", generator=gen))
    g.sub_(1).exp2_().mul_(1 + 2.0 ** -7 - 2.0 ** -12)
    g[:, -1] = 1 / 3
    gw, gb = torch.zeros((LONG_D, LONG_N), device="cuda"), torch.zeros(LONG_N, device="cuda")
    B.sat_mx_dense_tn(ctx, q, g, gw, gb)
    B.sat_sync_status(ctx)
    yield codes, g, gw, gb


def test_weight_gradient_of_a_million_rows_does_not_drift(long_gradient):
    """All terms are positive, so that what is chopped adds up.  A run of the leading accumulator is 24 instructions, two units of 2^-23 each at
    most; the accumulator of the lower terms, 2^-7 of the sum, is taken out every 384 stages of 4 instructions: 48 U + 2 * 1536 * 2^-7 U.  Runs are
    added up rounded to nearest: no drift, 0.3 U sqrt(2605 / 3) = 9 U to an element, 9 / 20 U in the mean of 400 independent ones."""
    import torch
    codes, g, gw, _ = long_gradient
    cols, rows = torch.linspace(0, LONG_D - 1, 40, device="cuda").long(), torch.linspace(0, LONG_N - 2, 10, device="cuda").long()
    c = codes[:, cols].long()
    a = (1 + (c % 8) / 8.0).double() * torch.exp2((c // 8 - 7).double())
    want = a.T @ g[:, rows].double()
    rel = (gw[cols][:, rows].double() - want) / want
    assert abs(float(rel.mean())) <= (48 + 2 * 1536 * 2.0 ** -7 + 6 * 9 / 20) * U
    assert float(rel.abs().max()) <= (48 + 2 * 1536 * 2.0 ** -7 + 6 * 9) * U


def test_bias_gradient_of_a_million_rows(long_gradient):
    """A thread adds up to 256 gradients before it adds that to a second sum, of at most a million / 8 / 256 = 489 terms: half a unit each."""
    _, g, _, gb = long_gradient
    want = g.double().sum(0)
    assert float(((gb.double() - want) / want).abs().max()) <= (256 + 489 + 4) * U / 2


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m,n,k", [(70, 100, 40000), (300, 33, 16385), (1, 1, 16384)])
def test_input_gradient_of_many_terms(B, ctx, bits, m, n, k):
    """The accumulators of the input gradient are read and begun anew several times.  Terms of one sign: a run of 32 instructions is off by two units each
    at most, the lower terms by 2048 instructions of theirs, 2^-7 of the sum, the runs by half a unit each."""
    rng = np.random.default_rng(k + bits)
    w = rng.choice([0.5, 1.0, 1.5, 2.0, 3.0], (k, n)).astype(np.float32)
    a = (2.0 ** rng.integers(-1, 2, (m, k)) * (1 + 2.0 ** -7 - 2.0 ** -12)).astype(np.float32)
    wq, wv = _mx(B, w, bits)
    out = _out(m, n)
    B.sat_mx_dense_nn(ctx, _dev(a), wq, out)
    B.sat_sync_status(ctx)
    want = a.astype(np.float64) @ wv
    assert np.all(np.abs(_np(out) - want) <= (64 + 2 * 2048 * 2.0 ** -7 + (k / 512 + 3) / 2) * U * want)
    a = _rows(rng, m, k)
    B.sat_mx_dense_nn(ctx, _dev(a), wq, out)
    B.sat_sync_status(ctx)
    assert np.all(np.abs(_np(out) - a.astype(np.float64) @ wv) <= _bound(a.astype(np.float64), wv, k))


@pytest.mark.parametrize("m", [1, 40])
def test_product_of_many_terms(B, ctx, m):
    """64 products an addition, in one accumulator (tiles) or a group at a time (a few rows)."""
    rng = np.random.default_rng(m)
    k, n = 92000, 45
    a, w = _rows(rng, m, k), rng.normal(size=(n, k)).astype(np.float32)
    aq, av = _mx(B, a, 4)
    wq, wv = _mx(B, w, 4)
    first, second = _out(m, n), _out(m, n)
    B.sat_mx_dense_nt(ctx, _dev(a), wq, None, first)
    B.sat_mx_dense_nt(ctx, aq, wq, None, second)
    B.sat_sync_status(ctx)
    assert np.array_equal(_np(first), _np(second))
    assert np.all(np.abs(_np(first) - av @ wv.T) <= _bound(av, wv.T, k))


@pytest.mark.parametrize("bits", [8, 4])
def test_rows_of_a_larger_matrix(B, ctx, bits):
    """Descriptions of a part of the rows: the others are left as they were and read by nobody."""
    import torch
    rng = np.random.default_rng(bits)
    a, g = _rows(rng, 500, 90), rng.normal(size=(500, 40)).astype(np.float32)
    whole, values = _mx(B, a, bits)
    codes, scales = whole._keep
    fmt = B.SAT_MX8 if bits == 8 else B.SAT_MX4
    part = B.make_mx(codes[133:400], scales[133:400], 90, fmt)
    gw, gb, gt = torch.zeros((90, 40), device="cuda"), torch.zeros(40, device="cuda"), _dev(g)
    B.sat_mx_dense_tn(ctx, part, gt[133:400], gw, gb)
    want = values[133:400].T @ g[133:400].astype(np.float64)
    assert np.all(np.abs(_np(gw) - want) <= _bound(values[133:400].T, g[133:400].astype(np.float64), 267))
    before = codes.clone(), scales.clone()
    B.sat_mx_quantise(ctx, _dev(2 * a)[133:400], part)
    B.sat_sync_status(ctx)
    c, s = mx.quantise(2 * a[133:400], bits)
    assert np.array_equal(codes[133:400].cpu().numpy()[:, :c.shape[1]], c) and np.array_equal(scales[133:400].cpu().numpy()[:, :s.shape[1]], s)
    for now, then in zip((codes, scales), before):
        assert bool(torch.equal(now[:133], then[:133])) and bool(torch.equal(now[400:], then[400:]))
