"""Microscaled matrices on the GPU against their 64-bit reference: codes and scales bit by bit, contractions within bounds that follow
from how they add.

Bounds.  A sum that keeps its running value in fp32 is off by at most one unit of 2^-23 of that value per addition (chopped) or half of it
(rounded), and the running value is at most S = sum |a| |b|.  sat_mx_dense_nt adds 64 exact products at a time: k / 64 + 1 additions, and as
many again for what is aligned inside one.  The other two have their fp32 operand in three exact terms and add 16 products at a time:
3 (k / 16 + 1) additions, the same again for alignment, and a few for joining partial sums.  CUDA-core forms round after every
product, k half units.  `_bound` takes the largest of these counts, which holds for every form.  Its 2-norm version (`_off`) is what signed
data show: errors of a chopped sum of T additions of random sign add up to about T / 3 units of its own size, and no form chops more
than 32 times in a row before it rounds: 32 / 3 * 2^-23 = 1.3e-6, with the rounded additions behind it below 2e-6.
"""
import numpy as np
import pytest

from oracle import mx_ref as mx

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.sat_create(0, 0)
    yield c
    B.sat_destroy(c)


def _rows(rng, rows, d, spread=1.0):
    """Rows of very different size with zeros in them, as ReLU layers leave them."""
    x = rng.normal(size=(rows, d)) * np.exp(spread * rng.normal(size=(rows, 1)))
    return np.where(rng.random((rows, d)) < 0.3, 0.0, x).astype(np.float32)


def _dev(a, extra=0, fill=float("nan")):
    """On the GPU with a row stride of round_up(d, 4) + extra floats; what lies between the rows is `fill`."""
    import torch
    rows, d = a.shape
    full = torch.full((max(rows, 1), (d + 3) // 4 * 4 + extra), fill, dtype=torch.float32, device="cuda")
    view = full[:rows, :d]
    view.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)))
    return view


def _out(rows, d, extra=0):
    return _dev(np.full((rows, d), 7.0, dtype=np.float32), extra)


def _mx(B, a, bits, extra=0):
    """The 64-bit reference's codes of `a` on the GPU (bytes behind the rows' ends are 0xA5 / 0xFF), and what they stand for."""
    import torch
    codes, scales = mx.quantise(a, bits)
    rows, d = a.shape
    ct = torch.full((rows, (codes.shape[1] + 15) // 16 * 16 + 16 * extra), 0xA5, dtype=torch.uint8, device="cuda")
    st = torch.full((rows, (scales.shape[1] + 3) // 4 * 4 + 4 * extra), 0xFF, dtype=torch.uint8, device="cuda")
    ct[:, :codes.shape[1]] = torch.from_numpy(codes).cuda()
    st[:, :scales.shape[1]] = torch.from_numpy(scales).cuda()
    return B.make_mx(ct, st, d, B.SAT_MX8 if bits == 8 else B.SAT_MX4), mx.dequantise(codes, scales, d, bits)


def _np(t):
    return t.detach().cpu().numpy().astype(np.float64)


def _bound(a, b, terms):
    """Per element: additions times a unit of sum |a| |b|."""
    return (terms / 2 + 6 * (terms / 16 + 1) + 8) * U * (np.abs(a) @ np.abs(b))


def _off(got, want):
    n = np.linalg.norm(want)
    return np.linalg.norm(got - want) / n if n else np.linalg.norm(got)


def _check(got, want, bound, loose=2e-6):
    assert got.shape == want.shape and np.isfinite(got).all()
    assert np.all(np.abs(got - want) <= bound + 1e-44), float(np.max(np.abs(got - want) - bound))
    assert _off(got, want) <= loose


def _untouched(view, d):
    """Nothing was written behind the rows' ends."""
    import torch
    full = view._base if view._base is not None else view
    return bool(torch.isnan(full[:view.shape[0], d:]).all())


# ---- quantisation ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,d,extra", [(1, 1, 0), (3, 31, 4), (7, 32, 0), (5, 33, 8), (129, 100, 0), (1000, 256, 4), (64, 602, 0), (2049, 7, 0), (2, 4099, 0), (9001, 257, 0), (8191, 290, 4), (76801, 30, 0), (9100, 256, 0)])
def test_codes_and_scales_bit_by_bit(B, ctx, bits, rows, d, extra):
    import torch
    rng = np.random.default_rng(rows * 7 + d)
    a = _rows(rng, rows, d, 3.0)
    want_c, want_s = mx.quantise(a, bits)
    ct = torch.full((rows, (want_c.shape[1] + 15) // 16 * 16 + 16), 0xA5, dtype=torch.uint8, device="cuda")
    st = torch.full((rows, (want_s.shape[1] + 3) // 4 * 4 + 4), 0xA5, dtype=torch.uint8, device="cuda")
    q = B.make_mx(ct, st, d, B.SAT_MX8 if bits == 8 else B.SAT_MX4)
    x = _dev(a, extra)
    B.sat_mx_quantise(ctx, x, q)
    B.sat_sync_status(ctx)
    c, s = ct.cpu().numpy(), st.cpu().numpy()
    assert np.array_equal(c[:, :want_c.shape[1]], want_c) and np.array_equal(s[:, :want_s.shape[1]], want_s)
    assert (c[:, want_c.shape[1]:] == 0xA5).all() and (s[:, want_s.shape[1]:] == 0xA5).all()
    y = _out(rows, d, extra)
    B.sat_mx_dequantise(ctx, q, y)
    B.sat_sync_status(ctx)
    assert np.array_equal(_np(y), mx.dequantise(want_c, want_s, d, bits)) and _untouched(y, d)


@pytest.mark.parametrize("bits", [8, 4])
def test_values_at_the_ends_of_the_range(B, ctx, bits):
    tiny, big = 2.0 ** -149, np.finfo(np.float32).max
    a = np.zeros((12, 64), dtype=np.float32)
    a[0, :4] = [tiny, -tiny, 3 * tiny, 2.0 ** -126]
    a[1, :4] = [big, -big, big / 2, 1.0]
    a[2, 5] = np.inf
    a[3, 6] = np.nan
    a[4, :3] = [-np.inf, np.nan, 1.0]
    a[5, :5] = [-0.0, 0.0, 1.0, -1e-30, 2.0 ** -127]
    a[6, :4] = [448.0, 449.0, 6.0, 6.5]
    a[7, :4] = [6.0, 5.0, 2.5, 0.25]
    a[8, :] = 2.0 ** -119 * np.linspace(-1, 1, 64)
    a[9, :] = 2.0 ** -125 * np.linspace(-1, 1, 64)
    a[10, 31], a[10, 32] = 1.75, 1.5
    a[11, :] = np.float32(2.0 ** 127)
    want_c, want_s = mx.quantise(a, bits)
    q = B.new_mx(12, 64, B.SAT_MX8 if bits == 8 else B.SAT_MX4)
    B.sat_mx_quantise(ctx, _dev(a), q)
    y = _out(12, 64)
    B.sat_mx_dequantise(ctx, q, y)
    B.sat_sync_status(ctx)
    assert np.array_equal(q._keep[0].cpu().numpy()[:, :want_c.shape[1]], want_c)
    assert np.array_equal(q._keep[1].cpu().numpy()[:, :2], want_s)
    want = mx.dequantise(want_c, want_s, 64, bits).astype(np.float32)
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)
    assert np.isnan(want[2, :32]).all() and not np.isnan(want[2, 32:]).any()


def test_places_beyond_32_bits(B, ctx):
    import torch
    rows, d = 70_000_000, 32                                      # 2.24 G elements
    x = torch.zeros((rows, d), device="cuda")
    rng = np.random.default_rng(0)
    tail = _rows(rng, 100, d)
    x[-100:] = torch.from_numpy(tail).cuda()
    q = B.new_mx(rows, d, B.SAT_MX8)
    B.sat_mx_quantise(ctx, x, q)
    x.fill_(5.0)
    B.sat_mx_dequantise(ctx, q, x)
    B.sat_sync_status(ctx)
    c, s = mx.quantise(tail, 8)
    assert np.array_equal(_np(x[-100:]), mx.dequantise(c, s, d, 8))
    assert not bool(x[:-100].any())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,d", [(58241, 602), (40000, 290), (150000, 64)])
def test_the_same_codes_every_time(B, ctx, bits, rows, d):
    """Passes behind one another, on matrices long enough that every stage of shared memory is filled many times."""
    import torch
    x = torch.randn((rows, (d + 3) // 4 * 4), device="cuda")[:, :d] * torch.exp(torch.randn((rows, 1), device="cuda"))
    x = x.contiguous() if d % 4 == 0 else torch.nn.functional.pad(x, (0, -d % 4))[:, :d]
    q, y = B.new_mx(rows, d, B.SAT_MX8 if bits == 8 else B.SAT_MX4), torch.zeros((rows, (d + 3) // 4 * 4), device="cuda")[:, :d]
    for t in q._keep:
        t.zero_()
    B.sat_mx_quantise(ctx, x, q)
    B.sat_mx_dequantise(ctx, q, y)
    part = np.r_[0:50, rows // 2:rows // 2 + 50, rows - 50:rows]
    c, s = mx.quantise(x.cpu().numpy()[part], bits)
    assert np.array_equal(q._keep[0].cpu().numpy()[part][:, :c.shape[1]], c) and np.array_equal(_np(y)[part], mx.dequantise(c, s, d, bits))
    first = [t.clone() for t in (*q._keep, y)]
    for _ in range(60):
        for t in (*q._keep, y):
            t.zero_()
        for _ in range(2):
            B.sat_mx_quantise(ctx, x, q)
            B.sat_mx_dequantise(ctx, q, y)
        assert all(bool(torch.equal(a, b)) for a, b in zip(first, (*q._keep, y)))


@pytest.mark.parametrize("m,n,k", [(60000, 256, 256), (30000, 100, 602)])
def test_the_same_results_every_time(B, ctx, m, n, k):
    import torch
    x, g = torch.randn((m, (k + 3) // 4 * 4), device="cuda")[:, :k], torch.randn((m, n), device="cuda")
    w8, w4, kept = B.new_mx(n, k, B.SAT_MX8), B.new_mx(n, k, B.SAT_MX4), B.new_mx(m, k, B.SAT_MX4)
    for t in (w8, w4):
        B.sat_mx_quantise(ctx, torch.nn.functional.pad(torch.randn((n, k), device="cuda"), (0, -k % 4))[:, :k], t)
    for t in kept._keep:
        t.zero_()
    y, gx, gw, gb = torch.zeros((m, n), device="cuda"), torch.zeros((m, (k + 3) // 4 * 4), device="cuda")[:, :k], torch.zeros((k, n), device="cuda"), torch.zeros(n, device="cuda")
    outs, first = (y, gx, gw, gb, *kept._keep), None
    for _ in range(40):
        for t in outs:
            t.zero_()
        for _ in range(2):
            B.sat_mx_dense_nt(ctx, x, w4, None, y, kept)
            B.sat_mx_dense_nn(ctx, g, w8, gx)
            B.sat_mx_dense_tn(ctx, kept, g, gw, gb)
        if first is None:
            first = [t.clone() for t in outs]
        assert all(bool(torch.equal(a, b)) for a, b in zip(first, outs))


# ---- contractions ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("m,n,k,extra", [(1, 1, 1, 0), (1, 512, 512, 0), (2, 40, 33, 4), (9, 17, 64, 0), (16, 130, 2050, 4), (33, 300, 129, 0), (127, 72, 50, 4), (128, 256, 256, 0),
                                         (129, 257, 31, 0), (1000, 47, 602, 0), (300, 600, 1030, 0), (4096, 128, 100, 0), (20000, 256, 256, 0), (19001, 40, 300, 4),
                                         (3001, 8, 64, 0), (301, 40, 10, 4), (40, 3, 2, 0), (5000, 1, 33, 0), (19, 1, 1, 0)])
@pytest.mark.parametrize("source", ["fp32", "kept", "codes"])
def test_product_of_4_bit_operands(B, ctx, m, n, k, extra, source):
    import torch
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    a, w, bias = _rows(rng, m, k), rng.normal(size=(n, k)).astype(np.float32), rng.normal(size=n).astype(np.float32)
    wq, wv = _mx(B, w, 4, extra)
    aq, av = _mx(B, a, 4, extra)
    out, bt = _out(m, n, extra), torch.from_numpy(bias).cuda()
    if source == "codes":
        B.sat_mx_dense_nt(ctx, aq, wq, bt, out)
    else:
        kept = B.new_mx(m, k, B.SAT_MX4) if source == "kept" else None
        B.sat_mx_dense_nt(ctx, _dev(a, extra), wq, bt, out, kept)
        if kept is not None:
            c, s = mx.quantise(a, 4)
            assert np.array_equal(kept._keep[0].cpu().numpy()[:, :c.shape[1]], c) and np.array_equal(kept._keep[1].cpu().numpy()[:, :s.shape[1]], s)
    B.sat_sync_status(ctx)
    want = av @ wv.T + bias
    _check(_np(out), want, _bound(av, wv.T, k) + U * (np.abs(want) + np.abs(bias)))
    assert _untouched(out, n)
    again = _out(m, n, extra)
    B.sat_mx_dense_nt(ctx, aq if source == "codes" else _dev(a, extra), wq, bt, again)
    assert bool(torch.equal(out, again))                           # the same bits every time
    B.sat_mx_dense_nt(ctx, aq if source == "codes" else _dev(a, extra), wq, None, again)
    _check(_np(again), av @ wv.T, _bound(av, wv.T, k))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m,n,k,extra", [(1, 1, 1, 0), (1, 512, 512, 0), (5, 33, 40, 4), (128, 256, 32, 0), (129, 100, 47, 0), (301, 100, 47, 4), (64, 257, 1000, 0), (1000, 600, 700, 0),
                                         (20000, 256, 40, 0), (19001, 300, 256, 4),
                                         (30001, 1, 413, 0), (20001, 7, 5, 4), (2630, 2, 570, 0), (40000, 33, 1, 0), (1, 448, 49, 0)])
def test_rows_times_stored_weights(B, ctx, bits, m, n, k, extra):
    import torch
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    a, w = _rows(rng, m, k, 2.0), rng.normal(size=(k, n)).astype(np.float32)
    wq, wv = _mx(B, w, bits, extra)
    out = _out(m, n, extra)
    B.sat_mx_dense_nn(ctx, _dev(a, extra), wq, out)
    B.sat_sync_status(ctx)
    _check(_np(out), a.astype(np.float64) @ wv, _bound(a.astype(np.float64), wv, k))
    assert _untouched(out, n)
    again = _out(m, n, extra)
    B.sat_mx_dense_nn(ctx, _dev(a, extra), wq, again)
    assert bool(torch.equal(out, again))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,m,n,extra", [(1, 1, 1, 0), (1, 300, 40, 0), (5, 33, 17, 4), (31, 64, 128, 0), (32, 256, 16, 0), (33, 100, 129, 0), (301, 100, 47, 4), (2048, 32, 16, 0),
                                            (1000, 602, 256, 0), (5000, 257, 130, 0), (30000, 256, 256, 4), (41001, 40, 300, 0),
                                            (20000, 64, 3, 0), (50001, 17, 192, 4), (30000, 1, 1, 0), (49, 1, 300, 4), (90, 300, 2, 0)])
def test_weight_and_bias_gradient_from_a_checkpoint(B, ctx, bits, rows, m, n, extra):
    import torch
    rng = np.random.default_rng(rows + 3 * m + 5 * n)
    a, g = _rows(rng, rows, m, 1.0), rng.normal(size=(rows, n)).astype(np.float32)
    aq, av = _mx(B, a, bits, extra)
    out, cs, gt = torch.full((m, n), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda"), _dev(g, extra)
    B.sat_mx_dense_tn(ctx, aq, gt, out, cs)
    B.sat_sync_status(ctx)
    g64 = g.astype(np.float64)
    want, want_cs = av.T @ g64, g64.sum(0)
    _check(_np(out), want, _bound(av.T, g64, rows))
    _check(_np(cs)[None], want_cs[None], _bound(np.ones((1, rows)), g64, rows))
    again, cs2 = torch.ones_like(out), torch.ones_like(cs)
    B.sat_mx_dense_tn(ctx, aq, gt, again, cs2)
    assert bool(torch.equal(out, again)) and bool(torch.equal(cs, cs2))
    B.sat_mx_dense_tn(ctx, aq, gt, again, cs2, accumulate=True)    # x + x
    _check(_np(again), 2 * want, 2 * _bound(av.T, g64, rows) + U * np.abs(want))
    _check(_np(cs2), 2 * want_cs, 2 * _bound(np.ones((1, rows)), g64, rows)[0] + U * np.abs(want_cs))
    B.sat_mx_dense_tn(ctx, aq, gt, again)
    assert bool(torch.equal(out, again))


def test_empty_operands(B, ctx):
    import torch
    e4, e8 = B.new_mx(0, 40, B.SAT_MX4), B.new_mx(0, 40, B.SAT_MX8)
    x0 = torch.zeros((0, 40), device="cuda")
    B.sat_mx_quantise(ctx, x0, e8)
    B.sat_mx_dequantise(ctx, e8, x0)
    out, cs = torch.full((40, 12), 3.0, device="cuda"), torch.full((12,), 3.0, device="cuda")
    B.sat_mx_dense_tn(ctx, e8, torch.zeros((0, 12), device="cuda"), out, cs, accumulate=True)
    assert bool((out == 3).all()) and bool((cs == 3).all())
    B.sat_mx_dense_tn(ctx, e4, torch.zeros((0, 12), device="cuda"), out, cs)
    assert not bool(out.any()) and not bool(cs.any())
    y = torch.full((5, 40), 3.0, device="cuda")
    B.sat_mx_dense_nn(ctx, torch.zeros((5, 0), device="cuda"), e4, y)
    assert not bool(y.any())
    w, _ = _mx(B, np.ones((8, 40), dtype=np.float32), 4)
    B.sat_mx_dense_nt(ctx, x0, w, None, torch.zeros((0, 8), device="cuda"))
    B.sat_mx_dense_nn(ctx, torch.zeros((0, 8), device="cuda"), w, x0)
    B.sat_sync_status(ctx)


def test_what_is_not_finite_reaches_its_results_and_no_others(B, ctx):
    import torch
    rng = np.random.default_rng(5)
    m, k, n = 300, 96, 72
    a, w = _rows(rng, m, k), rng.normal(size=(n, k)).astype(np.float32)
    a[17, 40] = np.inf
    a[200, 95] = np.nan
    w[5, 3] = np.nan
    wq, _ = _mx(B, w, 4)
    out = _out(m, n)
    B.sat_mx_dense_nt(ctx, _dev(a), wq, None, out)
    bad = np.zeros((m, n), dtype=bool)
    bad[[17, 200]] = True
    bad[:, 5] = True
    assert np.array_equal(np.isnan(_np(out)), bad)
    g = rng.normal(size=(m, n)).astype(np.float32)
    g[31, 8] = np.inf
    for bits in (8, 4):
        wq, _ = _mx(B, w, bits)
        gx = _out(m, k)
        B.sat_mx_dense_nn(ctx, _dev(g), wq, gx)                     # group 0 of row 5 of W is no number: columns 0 .. 31
        bad = np.zeros((m, k), dtype=bool)
        bad[31] = True
        bad[:, :32] = True
        assert np.array_equal(~np.isfinite(_np(gx)), bad)
        aq, _ = _mx(B, a, bits)
        gw = torch.zeros((k, n), device="cuda")
        B.sat_mx_dense_tn(ctx, aq, _dev(g), gw)
        bad = np.zeros((k, n), dtype=bool)
        bad[32:96] = True                                           # groups 1 (row 17) and 2 (row 200)
        bad[:, 8] = True
        assert np.array_equal(~np.isfinite(_np(gw)), bad)
    B.sat_sync_status(ctx)


@pytest.mark.parametrize("scale", [1e-36, 1e-18, 1e18, 1e34])
def test_operands_far_from_one(B, ctx, scale):
    import torch
    rng = np.random.default_rng(6)
    a, g = rng.normal(size=(700, 90)).astype(np.float32), (rng.normal(size=(700, 50)) * scale).astype(np.float32)
    aq, av = _mx(B, a, 8)
    out = torch.zeros((90, 50), device="cuda")
    B.sat_mx_dense_tn(ctx, aq, _dev(g), out)
    # bits of an fp32 element below 2^-133 are dropped: 2^-133 at most of each of 700 (50) products with an element up to 4, and 2^-133 / scale
    # relative to elements of that size
    loose = 2e-6 + 2.0 ** -133 / scale
    _check(_np(out), av.T @ g.astype(np.float64), _bound(av.T, g.astype(np.float64), 700) + 700 * 4 * 2.0 ** -133, loose)
    w = rng.normal(size=(50, 90)).astype(np.float32)
    wq, wv = _mx(B, w, 4)
    gx = _out(700, 90)
    B.sat_mx_dense_nn(ctx, _dev(g), wq, gx)
    _check(_np(gx), g.astype(np.float64) @ wv, _bound(g.astype(np.float64), wv, 50) + 50 * 4 * 2.0 ** -133, loose)
    x = (rng.normal(size=(700, 90)) * scale).astype(np.float32)
    xq, xv = _mx(B, x, 4)
    y = _out(700, 50)
    B.sat_mx_dense_nt(ctx, _dev(x), wq, None, y)
    _check(_np(y), xv @ wv.T, _bound(xv, wv.T, 90))


# ---- a layer trained on 4-bit operands --------------------------------------------------------------------------------------
def test_a_4_bit_layer_forward_and_backward(B, ctx):
    """y = x^ W^^T + b with x kept in 4 bits, L = sum R y: the gradients of the rounded operands are the formula's, and since L is linear in
    each of them, differences give them too."""
    import torch
    rng = np.random.default_rng(8)
    m, k, n = 777, 130, 70
    x, w, b, R = _rows(rng, m, k), rng.normal(size=(n, k)).astype(np.float32), rng.normal(size=n).astype(np.float32), rng.normal(size=(m, n)).astype(np.float32)
    wq = B.new_mx(n, k, B.SAT_MX4)
    B.sat_mx_quantise(ctx, _dev(w), wq)
    kept, y = B.new_mx(m, k, B.SAT_MX4), _out(m, n)
    B.sat_mx_dense_nt(ctx, _dev(x), wq, torch.from_numpy(b).cuda(), y, kept)
    gx, gwt, gb = _out(m, k), torch.zeros((k, n), device="cuda"), torch.zeros(n, device="cuda")
    B.sat_mx_dense_nn(ctx, _dev(R), wq, gx)
    B.sat_mx_dense_tn(ctx, kept, _dev(R), gwt, gb)
    B.sat_sync_status(ctx)
    xv, wv, R = mx.dequantise(*mx.quantise(x, 4), k, 4), mx.dequantise(*mx.quantise(w, 4), k, 4), R.astype(np.float64)
    _check(_np(y), xv @ wv.T + b, _bound(xv, wv.T, k) + U * (np.abs(xv @ wv.T + b) + np.abs(b)))
    _check(_np(gx), R @ wv, _bound(R, wv, n))
    _check(_np(gwt), xv.T @ R, _bound(xv.T, R, m))
    _check(_np(gb), R.sum(0), _bound(np.ones((1, m)), R, m)[0])
    loss = lambda xx, ww, bb: float(np.sum(R * (xx @ ww.T + bb)))
    for _ in range(10):
        i, j, o = rng.integers(m), rng.integers(k), rng.integers(n)
        dx, dw, db = np.zeros_like(xv), np.zeros_like(wv), np.zeros(n)
        dx[i, j], dw[o, j], db[o] = 0.5, 0.5, 0.5
        tol = 1e-3 * np.sqrt(m)
        assert abs(loss(xv + dx, wv, b) - loss(xv - dx, wv, b) - _np(gx)[i, j]) <= tol
        assert abs(loss(xv, wv + dw, b) - loss(xv, wv - dw, b) - _np(gwt)[j, o]) <= tol
        assert abs(loss(xv, wv, b + db) - loss(xv, wv, b - db) - _np(gb)[o]) <= tol


@pytest.mark.parametrize("rows", [1, 40, 3000])
def test_calls_captured_and_replayed_on_a_stream_of_their_own(B, rows):
    import torch
    rng = np.random.default_rng(rows)
    m, k, n = rows, 100, 72
    stream = torch.cuda.Stream()
    c = B.sat_create(0, stream.cuda_stream)
    try:
        with torch.cuda.stream(stream):
            x, g = _dev(_rows(rng, m, k)), _dev(rng.normal(size=(m, n)).astype(np.float32))
            wq, wv = _mx(B, rng.normal(size=(n, k)).astype(np.float32), 4)
            kept, y, gx, gw, gb, back = B.new_mx(m, k, B.SAT_MX4), _out(m, n), _out(m, k), torch.zeros((k, n), device="cuda"), torch.zeros(n, device="cuda"), _out(m, k)

            def step():
                B.sat_mx_dense_nt(c, x, wq, None, y, kept)
                B.sat_mx_dense_nn(c, g, wq, gx)
                B.sat_mx_dense_tn(c, kept, g, gw, gb)
                B.sat_mx_dequantise(c, kept, back)
            step()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step()
            for turn in range(2):
                a, r = _rows(rng, m, k), rng.normal(size=(m, n)).astype(np.float32)
                x.copy_(torch.from_numpy(a))
                g.copy_(torch.from_numpy(r))
                for t in (y, gx, gw, gb, back):
                    t.fill_(9.0)
                graph.replay()
                stream.synchronize()
                av, r = mx.dequantise(*mx.quantise(a, 4), k, 4), r.astype(np.float64)
                assert np.array_equal(_np(back), av)
                _check(_np(y), av @ wv.T, _bound(av, wv.T, k))
                _check(_np(gx), r @ wv, _bound(r, wv, n))
                _check(_np(gw), av.T @ r, _bound(av.T, r, m))
                _check(_np(gb), r.sum(0), _bound(np.ones((1, m)), r, m)[0])
            B.sat_sync_status(c)
            del graph
    finally:
        B.sat_destroy(c)


def test_refusals(B, ctx):
    import torch
    x = torch.zeros((40, 64), device="cuda")
    out = torch.full((40, 40), 2.0, device="cuda")
    q4, q8, w = B.new_mx(40, 64, B.SAT_MX4), B.new_mx(40, 64, B.SAT_MX8), B.new_mx(40, 64, B.SAT_MX4)

    def refused(call, *args, status=None):
        with pytest.raises(B.SatError) as e:
            call(ctx, *args)
        assert e.value.status == (B.SAT_EINVAL if status is None else status) and str(e.value)

    def changed(q, **kw):
        t = B.sat_mx_matrix(q.codes, q.scales, q.rows, q.d, q.ld_codes, q.ld_scales, q.format)
        t._keep = q._keep
        for k, v in kw.items():
            setattr(t, k, v)
        return t
    for kw in (dict(format=5), dict(ld_codes=q8.ld_codes + 8), dict(ld_codes=48), dict(ld_scales=0), dict(ld_scales=6), dict(codes=q8.codes + 8), dict(scales=q8.scales + 2),
               dict(codes=None), dict(scales=None)):
        refused(B.sat_mx_quantise, x, changed(q8, **kw))
        refused(B.sat_mx_dequantise, changed(q8, **kw), x)
        refused(B.sat_mx_dense_tn, changed(q8, **kw), x, torch.zeros((64, 64), device="cuda"))
        refused(B.sat_mx_dense_nn, out, changed(q8, **kw), x)
    refused(B.sat_mx_dense_nt, x, q8, None, out)                      # 8-bit weights
    refused(B.sat_mx_dense_nt, q8, w, None, out)                      # 8-bit rows
    refused(B.sat_mx_dense_nt, x, w, None, out, q8)
    refused(B.sat_mx_quantise, torch.zeros(40 * 64 + 1, device="cuda")[1:].view(40, 64), q4)
    refused(B.sat_mx_quantise, torch.zeros((40, 65), device="cuda")[:, :64], q4)
    refused(B.sat_mx_dense_nt, x, w, None, torch.zeros((40, 41), device="cuda")[:, :40])
    with pytest.raises(AssertionError):
        B.sat_mx_quantise(ctx, x[:39], q4)
    with pytest.raises(AssertionError):
        B.sat_mx_dense_nt(ctx, q4, w, None, out, q4)
    with pytest.raises(AssertionError):
        B.sat_mx_dense_tn(ctx, q4, x[:10], out)
    B.sat_sync_status(ctx)
    assert bool((out == 2).all())


def test_other_types_are_refused(B, ctx):
    import torch
    x, g, w = torch.zeros((40, 64), device="cuda"), torch.zeros((40, 8), device="cuda"), B.new_mx(8, 64, B.SAT_MX4)
    q, gw, gb, y = B.new_mx(40, 64, B.SAT_MX4), torch.zeros((64, 8), device="cuda"), torch.zeros(8, device="cuda"), torch.zeros((40, 8), device="cuda")
    for t in (torch.float64, torch.float16, torch.bfloat16, torch.int32):
        for call in (lambda: B.sat_mx_quantise(ctx, x.to(t), q), lambda: B.sat_mx_dequantise(ctx, q, x.to(t)), lambda: B.sat_mx_dense_nt(ctx, x.to(t), w, None, y),
                     lambda: B.sat_mx_dense_nt(ctx, x, w, gb.to(t), y), lambda: B.sat_mx_dense_nt(ctx, x, w, None, y.to(t)), lambda: B.sat_mx_dense_nn(ctx, g.to(t), w, x),
                     lambda: B.sat_mx_dense_nn(ctx, g, w, x.to(t)), lambda: B.sat_mx_dense_tn(ctx, q, g.to(t), gw), lambda: B.sat_mx_dense_tn(ctx, q, g, gw.to(t)),
                     lambda: B.sat_mx_dense_tn(ctx, q, g, gw, gb.to(t))):
            with pytest.raises(AssertionError):
                call()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,d,extra", [(310001, 1, 0), (310000, 3, 4), (160000, 33, 0), (155000, 61, 4), (110000, 66, 0), (152000, 64, 8)])
def test_long_matrices_back_to_fp32(B, ctx, bits, rows, d, extra):
    """Widths whose last elements fill no 16 bytes: every value exact, nothing written behind a row's end."""
    import torch
    a = _rows(np.random.default_rng(rows + d), rows, d, 3.0)
    q, values = _mx(B, a, bits)
    out = _out(rows, d, extra)
    B.sat_mx_dequantise(ctx, q, out)
    B.sat_sync_status(ctx)
    assert np.array_equal(_np(out), values.astype(np.float32)) and _untouched(out, d)
    again = B.new_mx(rows, d, B.SAT_MX8 if bits == 8 else B.SAT_MX4)
    B.sat_mx_quantise(ctx, _dev(a, extra), again)
    second = _out(rows, d, extra)
    B.sat_mx_dequantise(ctx, again, second)
    assert bool(torch.equal(out, second))
