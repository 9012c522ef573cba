"""Layer norm, forward and backward, against its definition in 64 bits.

Tolerances.  U = 2^-24 is fp32's half step.  A sum over a row of up to 16,384 terms is made of at most 16 terms a thread, five lane steps and five
warp steps in fp32 (32 terms a lane at most in rows of up to 256 pieces of 16 bytes): below 48 additions one after the other, so a mean is off by at most
48 U times the mean magnitude of its terms.
  forward   x - mean is off by that (the part of the mean's rounding that is seen again is taken off) and by U |x - mean| for each of two roundings; s by
            half of the variance's 50 U: |xh| by 64 U (1 + |xh|) with room to spare, and y by two more roundings and the type's own.
  backward  xh, from given mean and s, by 2 U |xh|; u by U; the two means by 52 U of theirs; all in all 64 U s (|u| + mean |u| + |xh| mean |u xh|)
  sums      over the rows of a block, the rows held side by side in it, the blocks: below 300 additions, each term off by 3 U
"""
import numpy as np
import pytest

from oracle import rows_ref as ref
from tests.rows_util import GUARD, HALF, U, dtype, guarded, host, matrix, room, rounding, within

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [(1, 1), (3, 7), (1, 8), (33, 16), (64, 32), (100, 50), (257, 100), (5, 128), (300, 256), (77, 602), (19, 1000), (9, 1025), (1, 2048), (6, 2050), (5, 4100),
          (3, 8192), (2, 10007), (2, 16384), (20000, 24)]


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.sat_create(0, 0)
    yield c
    B.sat_destroy(c)


def _vec(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def _inputs(rows, d, t, seed, extra=1):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, d)) * np.exp(rng.normal(size=(rows, 1))) + rng.normal(size=(rows, 1))
    g = rng.normal(size=(rows, d)) * np.exp(rng.normal(size=(rows, 1)))
    gamma, beta = (1 + 0.3 * rng.normal(size=d)).astype(np.float32), rng.normal(size=d).astype(np.float32)
    return matrix(x, t, extra)[0], matrix(g, t, extra)[0], gamma, beta


def _check_forward(x, gamma, beta, eps, y, mean, rstd, t):
    xd = host(x)
    want, m, s = ref.norm_fwd(xd, 1.0 if gamma is None else gamma.astype(np.float64), 0.0 if beta is None else beta.astype(np.float64), eps)
    ga, be = (np.abs(np.ones(1) if gamma is None else gamma), np.abs(np.zeros(1) if beta is None else beta))
    xh = np.abs(xd - m[:, None]) * s[:, None]
    within(host(y), want, ga * 64 * U * (1 + xh) + 2 * U * (ga * xh + be) + rounding(want, t) * 1.01, "y")
    within(host(mean), m, 50 * U * np.abs(xd - m[:, None]).mean(1) + U * np.abs(m) + 1e-45, "mean")
    within(host(rstd), s, 32 * U * s, "rstd")
    return m, s


def _check_backward(x, g, gamma, mean, rstd, g_x, g_gamma, g_beta, t, old=0.0):
    xd, gd, ga = host(x), host(g), np.ones(x.shape[1]) if gamma is None else gamma.astype(np.float64)
    m, s = host(mean), host(rstd)
    want, want_gamma, want_beta = ref.norm_bwd(xd, gd, ga, m, s)
    xh, u = (xd - m[:, None]) * s[:, None], gd * ga
    if g_x is not None:
        mag = np.abs(u) + np.abs(u).mean(1, keepdims=True) + np.abs(xh) * np.abs(u * xh).mean(1, keepdims=True)
        within(host(g_x), want, 64 * U * s[:, None] * mag + rounding(want, t) * 1.01, "g_x")
    for got, sums, mag in ((g_gamma, want_gamma, np.abs(gd * xh).sum(0)), (g_beta, want_beta, np.abs(gd).sum(0))):
        if got is not None:
            within(host(got), sums + old, 303 * U * mag + 2 * U * np.abs(sums + old) + 1e-45, "sums over the rows")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d", SHAPES)
def test_forward_and_backward(B, ctx, rows, d, t):
    import torch
    x, g, gamma, beta = _inputs(rows, d, t, rows + d)
    y, yf = room(rows, d, t, extra=2)
    g_x, gxf = room(rows, d, t)
    mean, rstd = (torch.full((rows,), np.nan, device="cuda") for _ in range(2))
    g_gamma, g_beta = torch.full((d,), np.nan, device="cuda"), torch.full((d,), np.nan, device="cuda")
    B.sat_layernorm_fwd(ctx, x, _vec(gamma), _vec(beta), EPS, y, mean, rstd)
    B.sat_layernorm_bwd(ctx, x, g, _vec(gamma), mean, rstd, g_x, g_gamma, g_beta)
    B.sat_sync_status(ctx)
    _check_forward(x, gamma, beta, EPS, y, mean, rstd, t)
    _check_backward(x, g, gamma, mean, rstd, g_x, g_gamma, g_beta, t)
    assert guarded(yf, d) and guarded(gxf, d)
    again = [v.clone() for v in (y, g_x, g_gamma, g_beta)]                      # the same bits
    B.sat_layernorm_fwd(ctx, x, _vec(gamma), _vec(beta), EPS, y, mean, rstd)
    B.sat_layernorm_bwd(ctx, x, g, _vec(gamma), mean, rstd, g_x, g_gamma, g_beta)
    for a, b in zip(again, (y, g_x, g_gamma, g_beta)):
        assert torch.equal(a, b)
    old = 3.0                                                                   # added to what is there
    g_gamma.fill_(old)
    g_beta.fill_(old)
    B.sat_layernorm_bwd(ctx, x, g, _vec(gamma), mean, rstd, None, g_gamma, g_beta, accumulate=True)
    _check_backward(x, g, gamma, mean, rstd, None, g_gamma, g_beta, t, old)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", [(40, 33), (9, 300), (3, 5000)])
def test_without_parameters_and_in_place(B, ctx, rows, d, t):
    import torch
    x, g, gamma, beta = _inputs(rows, d, t, 7 * rows + d)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y = room(rows, d, t)[0]
    B.sat_layernorm_fwd(ctx, x, None, None, EPS, y, mean, rstd)
    _check_forward(x, None, None, EPS, y, mean, rstd, t)
    g_x, g_beta = room(rows, d, t)[0], torch.empty(d, device="cuda")
    B.sat_layernorm_bwd(ctx, x, g, None, mean, rstd, g_x, None, g_beta)
    _check_backward(x, g, None, mean, rstd, g_x, None, g_beta, t)
    for place in (g.clone(), x.clone()):                                        # g_x in the place of g, and of x
        full, _ = room(rows, d, t)
        full.copy_(place)
        a, b = (x, full) if torch.equal(place, g) else (full, g)
        B.sat_layernorm_bwd(ctx, a, b, None, mean, rstd, full)
        assert torch.equal(full, g_x)
    same, _ = room(rows, d, t)                                                  # y in the place of x, no statistics kept
    same.copy_(x)
    B.sat_layernorm_fwd(ctx, same, None, None, EPS, same)
    assert torch.equal(same, y)
    B.sat_sync_status(ctx)


@pytest.mark.parametrize("d", [8, 100, 1500, 5000])
def test_rows_with_offsets_constants_and_no_numbers(B, ctx, d):
    import torch
    rng = np.random.default_rng(d)
    x = rng.normal(size=(9, d))
    x[1] += 1e4
    x[2] = 37.1
    x[3] = 0.0
    x[4] *= 1e12
    x[5, d // 2] = np.inf
    x[6, d - 1] = np.nan
    x[7] *= 1e-12
    xt = matrix(x, "f32", 1)[0]
    y, g_x = room(9, d, "f32")[0], room(9, d, "f32")[0]
    mean, rstd = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    B.sat_layernorm_fwd(ctx, xt, None, None, EPS, y, mean, rstd)
    bad = np.zeros(9, dtype=bool)
    bad[[5, 6]] = True
    assert np.isnan(host(y)[bad]).all() and np.isfinite(host(y)[~bad]).all()
    keep = torch.from_numpy(~bad).cuda()
    _check_forward(xt[keep], None, None, EPS, y[keep], mean[keep], rstd[keep], "f32")
    g = matrix(rng.normal(size=(9, d)), "f32")[0]
    B.sat_layernorm_bwd(ctx, xt, g, None, mean, rstd, g_x)
    assert np.isnan(host(g_x)[bad]).any(1).all()
    _check_backward(xt[keep], g[keep], None, mean[keep], rstd[keep], g_x[keep], None, None, "f32")
    B.sat_sync_status(ctx)


def test_no_rows(B, ctx):
    import torch
    x, g, gamma, beta = _inputs(1, 40, "f32", 1)
    g_gamma, g_beta, none = torch.full((40,), 2.0, device="cuda"), torch.full((40,), 2.0, device="cuda"), torch.empty(0, device="cuda")
    B.sat_layernorm_fwd(ctx, x[:0], _vec(gamma), None, EPS, x[:0], none, none)
    B.sat_layernorm_bwd(ctx, x[:0], g[:0], _vec(gamma), none, none, g[:0], g_gamma, g_beta, accumulate=True)
    assert bool((g_gamma == 2).all()) and bool((g_beta == 2).all())
    B.sat_layernorm_bwd(ctx, x[:0], g[:0], _vec(gamma), none, none, g[:0], g_gamma, g_beta)
    assert bool((g_gamma == 0).all()) and bool((g_beta == 0).all())
    B.sat_sync_status(ctx)


def test_offsets_beyond_32_bits(B, ctx):
    """Rows so far apart that the last ones lie more than 2^31 elements behind the first."""
    import torch
    rows, d, ld = 70000, 12, 32768
    big = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")
    x = big[:, :d]
    x.normal_()
    keep = x.clone()
    want = room(rows, d, "bf16")[0]
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    g_x, near = room(rows, d, "bf16")[0], room(rows, d, "bf16")[0]
    near.copy_(keep)
    B.sat_layernorm_fwd(ctx, near, None, None, EPS, want)
    B.sat_layernorm_bwd(ctx, near, near, None, mean.fill_(0.1), rstd.fill_(1.1), g_x)
    B.sat_layernorm_bwd(ctx, x, near, None, mean, rstd, near)
    assert torch.equal(near, g_x)
    B.sat_layernorm_fwd(ctx, x, None, None, EPS, x)
    assert torch.equal(x, want)
    B.sat_sync_status(ctx)


def test_on_a_side_stream_and_in_a_graph(B):
    import torch
    stream = torch.cuda.Stream()
    ctx = B.sat_create(0, stream.cuda_stream)
    try:
        x, g, gamma, beta = _inputs(500, 100, "f32", 5)
        ga, be = _vec(gamma), _vec(beta)
        y, g_x = room(500, 100, "f32")[0], room(500, 100, "f32")[0]
        mean, rstd, gg, gb = torch.empty(500, device="cuda"), torch.empty(500, device="cuda"), torch.empty(100, device="cuda"), torch.empty(100, device="cuda")
        torch.cuda.synchronize()

        def both():
            B.sat_layernorm_fwd(ctx, x, ga, be, EPS, y, mean, rstd)
            B.sat_layernorm_bwd(ctx, x, g, ga, mean, rstd, g_x, gg, gb)

        with torch.cuda.stream(stream):
            both()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                both()
            x2, g2, _, _ = _inputs(500, 100, "f32", 6)
            x.copy_(x2)
            g.copy_(g2)
            for t in (y, g_x, mean, rstd, gg, gb):
                t.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
        _check_forward(x, gamma, beta, EPS, y, mean, rstd, "f32")
        _check_backward(x, g, gamma, mean, rstd, g_x, gg, gb, "f32")
        del graph
    finally:
        B.sat_destroy(ctx)


def test_refusals(B, ctx):
    """Arguments that make no call: an error status, nothing launched, outputs as they were."""
    import torch
    x, g, gamma, beta = _inputs(10, 20, "f32", 3)
    y, mean, rstd, gg = room(10, 20, "f32")[0], torch.empty(10, device="cuda"), torch.empty(10, device="cuda"), torch.full((20,), 5.0, device="cuda")
    y.fill_(4.0)
    p, lib = (lambda t: None if t is None else t.data_ptr()), B._lib
    before = B.sat_launch_count(ctx)
    F = lambda rows=10, d=20, t=0, x=p(x), ld=24, ga=None, be=None, eps=EPS, y=p(y), ldy=24: lib.sat_layernorm_fwd(ctx, rows, d, t, x, ld, ga, be, eps, y, ldy, None, None)
    for bad in (F(t=3), F(t=-1), F(rows=-1), F(rows=2 ** 31), F(d=0), F(d=16385, ld=16388, ldy=16388), F(x=None), F(y=None), F(x=p(x) + 4), F(y=p(y) + 8), F(ld=19), F(ld=22),
                F(ldy=16), F(t=1, ld=20), F(eps=-1.0), F(eps=float("nan")), F(ga=p(gg) + 4), F(be=p(gg) + 4)):
        assert bad == B.SAT_EINVAL
    K = lambda rows=10, d=20, t=0, x=p(x), g=p(g), m=p(mean), s=p(rstd), gx=p(y), ldx=24, gg=p(gg), acc=0: lib.sat_layernorm_bwd(ctx, rows, d, t, x, 24, g, 24, None, m, s, gx, ldx, gg, None, acc)
    for bad in (K(t=7), K(rows=-2), K(d=0), K(x=None), K(g=None), K(m=None), K(s=None), K(gx=p(y) + 4), K(ldx=21), K(gx=None, gg=None), K(acc=2), K(g=p(g) + 4)):
        assert bad == B.SAT_EINVAL
    assert B.sat_launch_count(ctx) == before and bool((y == 4).all()) and bool((gg == 5).all())
    with pytest.raises(B.SatError):
        B.sat_layernorm_fwd(ctx, x, None, None, -1.0, y)
    for wrong in (lambda: B.sat_layernorm_fwd(ctx, x.double(), None, None, EPS, y), lambda: B.sat_layernorm_fwd(ctx, x, None, None, EPS, y[:5]),
                  lambda: B.sat_layernorm_fwd(ctx, x, gg[:19], None, EPS, y), lambda: B.sat_layernorm_fwd(ctx, x, gg.half(), None, EPS, y),
                  lambda: B.sat_layernorm_fwd(ctx, x, None, None, EPS, y.half()), lambda: B.sat_layernorm_fwd(ctx, x.t(), None, None, EPS, y.t()),
                  lambda: B.sat_layernorm_fwd(ctx, x.cpu(), None, None, EPS, y), lambda: B.sat_layernorm_bwd(ctx, x, g, None, mean[:9], rstd, y)):
        with pytest.raises(AssertionError):
            wrong()
    B.sat_sync_status(ctx)
