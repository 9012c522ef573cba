"""Embedding lookup, the order of a batch of tokens and the table's gradient, against their definitions.

The order is made of whole numbers and has to be equal, the lookup is one product rounded once.  Gradients: U = 2^-24 is fp32's half step; a token's c
rows are added in runs of at most 25 positions at these sizes, twice that where it crosses one border, the runs' sums up to 31 one after the other or by 32 threads and more side
by side: below 64 + c / 256 additions one after the other, and two more roundings.
"""
import numpy as np
import pytest

from oracle import rows_ref as ref
from tests.rows_util import U, guarded, host, matrix, room, rounding, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.sat_create(0, 0)
    yield c
    B.sat_destroy(c)


def _ints(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _tokens(rng, n, vocabulary, kind):
    if kind == "even":
        t = rng.integers(0, vocabulary, n)
    elif kind == "few":                                                         # the i-th about as often as 1 / i
        t = np.minimum(np.exp(rng.random(n) * np.log(vocabulary + 1)).astype(np.int64) - 1, vocabulary - 1)
    elif kind == "one":
        t = np.full(n, vocabulary - 1)
    else:                                                                       # every token once, then some again
        t = np.concatenate([rng.permutation(vocabulary)[:n], rng.integers(0, vocabulary, max(0, n - vocabulary))])
    return t.astype(np.int32)


CASES = [(1, 1, "even"), (1, 5000, "even"), (31, 2, "even"), (32, 16, "even"), (33, 1, "one"), (64, 7, "one"), (100, 40, "few"), (2048, 16, "even"), (4095, 300, "few"),
         (4096, 2047, "even"), (4097, 2048, "few"), (9000, 3, "one"), (20000, 5000, "few"), (30000, 20000, "each"), (50000, 612257, "few"), (70000, 64, "few")]


@pytest.mark.parametrize("n,vocabulary,kind", CASES + [(5000, 2 ** 22 + 5, "even"), (3000, 2 ** 31 - 2, "ends")])
@pytest.mark.parametrize("padding", [-1, 0])
def test_order(B, ctx, n, vocabulary, kind, padding):
    rng = np.random.default_rng(n + vocabulary)
    t = rng.choice(np.array([1, 5, 2 ** 30, vocabulary - 1, vocabulary - 2], dtype=np.int32), n) if kind == "ends" else _tokens(rng, n, vocabulary, kind)
    order = B.new_token_order(n, vocabulary)
    B.sat_token_sort(ctx, _ints(t), padding, order)
    B.sat_sync_status(ctx)
    tokens, index = order._keep
    for got, want in zip((tokens, index), ref.token_order(t, padding, vocabulary)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_tokens_outside_the_vocabulary(B, ctx):
    import torch
    rng = np.random.default_rng(0)
    t = rng.integers(0, 50, 6000).astype(np.int32)
    t[::7], t[3::100], t[5::90] = -1, 50, 2 ** 31 - 1
    t[11::50] = -5
    tab, _ = matrix(rng.normal(size=(50, 20)), "f32")
    out, full = room(6000, 20, "f32", 1)
    B.sat_embed_fwd(ctx, _ints(t), tab, 1.0, -1, out)
    with pytest.raises(B.SatError) as e:
        B.sat_sync_status(ctx)
    assert e.value.status == B.SAT_EDATA and "token" in str(e.value)
    B.sat_sync_status(ctx)                                                      # said once
    assert np.array_equal(host(out), ref.embed_fwd(t, host(tab), 1.0, -1)) and guarded(full, 20)
    order = B.new_token_order(6000, 50)
    B.sat_token_sort(ctx, _ints(t), -1, order)
    with pytest.raises(B.SatError) as e:
        B.sat_sync_status(ctx)
    assert e.value.status == B.SAT_EDATA
    for got, want in zip(order._keep, ref.token_order(t, -1, 50)):
        assert np.array_equal(got.cpu().numpy(), want)
    g, _ = matrix(rng.integers(-8, 9, (6000, 20)), "f32")                       # sums that fp32 holds
    gt = torch.full((50, 20), np.nan, device="cuda")
    B.sat_embed_bwd(ctx, order, g, 0.5, gt)
    B.sat_sync_status(ctx)
    assert np.array_equal(host(gt), ref.embed_bwd(t, host(g), 0.5, -1, 50)[0])
    only = np.full(100, 3, dtype=np.int32)                                      # nothing but padding
    order = B.new_token_order(100, 50)
    B.sat_token_sort(ctx, _ints(only), 3, order)
    B.sat_embed_bwd(ctx, order, g[:100], 0.5, gt)
    B.sat_sync_status(ctx)
    assert bool((gt == 0).all())


def test_an_order_that_is_none(B, ctx):
    """The arrays are the caller's: positions that the batch does not have are told apart from others, and nothing is read there."""
    import torch
    order = B.new_token_order(40, 9)
    tokens, index = order._keep
    tokens.copy_(_ints(np.sort(np.arange(40) % 9)))
    index.copy_(_ints(np.arange(40)))
    index[7], index[20] = 40, -3
    g, gt = matrix(np.ones((40, 8)), "f32")[0], torch.zeros((9, 8), device="cuda")
    B.sat_embed_bwd(ctx, order, g, 1.0, gt)
    with pytest.raises(B.SatError) as e:
        B.sat_sync_status(ctx)
    assert e.value.status == B.SAT_EDATA
    assert float(gt.sum()) == 38 * 8


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,vocabulary,d,kind", [(1, 1, 1, "even"), (50, 7, 3, "even"), (300, 40, 32, "few"), (1000, 100, 50, "few"), (257, 612257, 100, "even"), (40, 9, 602, "even"),
                                                 (33, 4, 4100, "few"), (20000, 5000, 16, "few")])
def test_lookup(B, ctx, n, vocabulary, d, kind, t):
    rng = np.random.default_rng(n + d)
    tokens, scale = _tokens(rng, n, vocabulary, kind), float(np.float32(np.sqrt(d)))
    table, _ = matrix(rng.normal(size=(vocabulary, d)), t, 1)
    out, full = room(n, d, t, 2)
    for padding in (-1, int(tokens[0])):
        B.sat_embed_fwd(ctx, _ints(tokens), table, scale, padding, out)
        B.sat_sync_status(ctx)
        want = ref.embed_fwd(tokens, host(table), scale, padding)
        within(host(out), want, rounding(want, t) + U * np.abs(want), "rows")
        assert guarded(full, d)
        B.sat_embed_fwd(ctx, _ints(tokens), table, 1.0, padding, out)
        assert np.array_equal(host(out), ref.embed_fwd(tokens, host(table), 1.0, padding))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [1, 8, 30, 50, 100, 130, 602])
@pytest.mark.parametrize("n,vocabulary,kind", [c for c in CASES if c[0] * 100 <= 3e6])
def test_gradient(B, ctx, n, vocabulary, kind, d, t):
    import torch
    if vocabulary * d > 6e7 or n * d > 8e6:
        d = 30
    rng = np.random.default_rng(n + vocabulary + d)
    tokens, scale = _tokens(rng, n, vocabulary, kind), 1.7
    g, _ = matrix(rng.normal(size=(n, d)) * np.exp(rng.normal(size=(n, 1))), t, 1)
    padding = int(tokens[n // 2]) if n > 60 and kind != "one" else -1
    order = B.new_token_order(n, vocabulary)
    B.sat_token_sort(ctx, _ints(tokens), padding, order)
    gt, full = room(vocabulary, d, "f32", 1)
    B.sat_embed_bwd(ctx, order, g, scale, gt)
    B.sat_sync_status(ctx)
    want, mag = ref.embed_bwd(tokens, host(g), float(np.float32(scale)), padding, vocabulary)
    count = np.bincount(tokens, minlength=vocabulary)[:, None]
    tol = (66 + count / 256) * U * mag
    within(host(gt), want, tol, "gradient")
    none = torch.from_numpy(mag.sum(1) == 0).cuda()
    assert guarded(full, d) and bool((gt[none] == 0).all())
    first = gt.clone()
    B.sat_embed_bwd(ctx, order, g, scale, gt)
    assert torch.equal(first, gt)                                               # the same bits
    gt.fill_(2.5)
    B.sat_embed_bwd(ctx, order, g, scale, gt, accumulate=True)
    B.sat_sync_status(ctx)
    within(host(gt), want + 2.5, tol + U * np.abs(want + 2.5), "added")
    assert guarded(full, d) and bool((gt[none] == 2.5).all())


def test_one_order_for_two_tables(B, ctx):
    import torch
    rng = np.random.default_rng(4)
    tokens = _tokens(rng, 3000, 90, "few")
    order = B.new_token_order(3000, 90)
    B.sat_token_sort(ctx, _ints(tokens), -1, order)
    for d, t in ((24, "f32"), (72, "bf16")):
        g, _ = matrix(rng.normal(size=(3000, d)), t)
        gt = torch.empty((90, d), device="cuda")
        B.sat_embed_bwd(ctx, order, g, 1.0, gt)
        want, mag = ref.embed_bwd(tokens, host(g), 1.0, -1, 90)
        within(host(gt), want, (66 + 3000 / 256) * U * mag, "gradient")
    B.sat_sync_status(ctx)


def test_no_tokens(B, ctx):
    import torch
    order, gt = B.new_token_order(0, 6), torch.full((6, 8), 2.0, device="cuda")
    none, rows = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 8), device="cuda")
    B.sat_token_sort(ctx, none, -1, order)
    B.sat_embed_bwd(ctx, order, rows, 1.0, gt, accumulate=True)
    assert bool((gt == 2).all())
    B.sat_embed_bwd(ctx, order, rows, 1.0, gt)
    assert bool((gt == 0).all())
    B.sat_embed_fwd(ctx, none, gt, 1.0, -1, rows)
    B.sat_sync_status(ctx)


def test_offsets_beyond_32_bits(B, ctx):
    """Gradient rows and table rows whose last ones lie more than 2^31 elements behind the first."""
    import torch
    n, d, ld = 70000, 8, 32768
    big = torch.empty((n, ld), dtype=torch.bfloat16, device="cuda")
    g = big[:, :d]
    g.copy_(torch.randint(-4, 5, (n, d), device="cuda"))
    near = g.contiguous()
    tokens = torch.randint(0, n, (n,), device="cuda", dtype=torch.int32)
    tokens[-1] = n - 1
    order = B.new_token_order(n, n)
    B.sat_token_sort(ctx, tokens, -1, order)
    a, b = torch.empty((n, d), device="cuda"), torch.empty((n, d), device="cuda")
    B.sat_embed_bwd(ctx, order, g, 1.0, a)
    B.sat_embed_bwd(ctx, order, near, 1.0, b)
    assert torch.equal(a, b)
    want = torch.zeros((n, d), device="cuda").index_add_(0, tokens.long(), near.float())
    assert torch.equal(a, want)                                                 # whole numbers: any order of addition
    out, out2 = torch.empty((n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    B.sat_embed_fwd(ctx, tokens, g, 2.0, -1, out)
    B.sat_embed_fwd(ctx, tokens, near, 2.0, -1, out2)
    assert torch.equal(out, out2) and torch.equal(out, 2 * near[tokens.long()])
    B.sat_sync_status(ctx)


def test_on_a_side_stream_and_in_a_graph(B):
    import torch
    stream = torch.cuda.Stream()
    ctx = B.sat_create(0, stream.cuda_stream)
    try:
        n, v, d = 5000, 700, 40
        tokens = torch.randint(0, v, (n,), device="cuda", dtype=torch.int32)
        g, order, gt = torch.randint(-9, 9, (n, d), device="cuda").float(), B.new_token_order(n, v), torch.empty((v, d), device="cuda")
        torch.cuda.synchronize()

        def both():
            B.sat_token_sort(ctx, tokens, -1, order)
            B.sat_embed_bwd(ctx, order, g, 1.0, gt)

        with torch.cuda.stream(stream):
            both()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                both()
            tokens.copy_(torch.randint(0, 30, (n,), device="cuda", dtype=torch.int32))
            gt.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
        assert torch.equal(gt, torch.zeros((v, d), device="cuda").index_add_(0, tokens.long(), g))
        del graph
    finally:
        B.sat_destroy(ctx)


def test_refusals(B, ctx):
    import torch
    rng = np.random.default_rng(0)
    table, out, tokens = matrix(rng.normal(size=(9, 20)), "f32")[0], room(5, 20, "f32")[0], _ints(np.zeros(5))
    out.fill_(4.0)
    lib, p = B._lib, lambda t: t.data_ptr()
    before = B.sat_launch_count(ctx)
    F = lambda n=5, t=p(tokens), v=9, d=20, ty=0, tab=p(table), ld=20, o=p(out), ldo=20: lib.sat_embed_fwd(ctx, n, t, v, -1, d, ty, tab, ld, 1.0, o, ldo)
    for bad in (F(n=-1), F(n=2 ** 31), F(t=None), F(v=0), F(v=-3), F(v=2 ** 31 - 1), F(d=0), F(d=21), F(ty=9), F(tab=None), F(tab=p(table) + 4), F(ld=18), F(ty=1), F(o=None), F(o=p(out) + 4),
                F(ldo=22)):
        assert bad == B.SAT_EINVAL
    order = B.new_token_order(5, 9)
    gt = torch.full((9, 20), 5.0, device="cuda")
    import ctypes as C
    S = lambda o, t=p(tokens): lib.sat_token_sort(ctx, t, -1, None if o is None else C.byref(o))
    K = lambda o=order, d=20, ty=0, g=p(out), ld=20, t=p(gt), ldt=20, acc=0: lib.sat_embed_bwd(ctx, None if o is None else C.byref(o), d, ty, g, ld, 1.0, t, ldt, acc)

    def changed(**kw):
        o = B.sat_token_order(order.tokens, order.index, order.n, order.vocabulary)
        for k, v in kw.items():
            setattr(o, k, v)
        return o

    for o in (None, changed(tokens=None), changed(index=None), changed(n=-1), changed(n=2 ** 31), changed(vocabulary=0), changed(vocabulary=2 ** 31 - 1)):
        assert S(o) == B.SAT_EINVAL and K(o=o) == B.SAT_EINVAL
    assert S(order, None) == B.SAT_EINVAL and S(order, order.tokens) == B.SAT_EINVAL and S(order, order.index) == B.SAT_EINVAL
    for bad in (K(d=0), K(d=21), K(ty=5), K(g=None), K(g=p(out) + 8), K(ld=22), K(t=None), K(t=p(gt) + 4), K(ldt=16), K(acc=3), K(ty=2)):
        assert bad == B.SAT_EINVAL
    assert B.sat_launch_count(ctx) == before and bool((gt == 5).all()) and bool((out == 4).all())
    for wrong in (lambda: B.sat_embed_fwd(ctx, tokens.long(), table, 1.0, -1, out), lambda: B.sat_embed_fwd(ctx, tokens[:4], table, 1.0, -1, out),
                  lambda: B.sat_embed_fwd(ctx, tokens, table.half(), 1.0, -1, out), lambda: B.sat_embed_fwd(ctx, tokens.cpu(), table, 1.0, -1, out),
                  lambda: B.sat_token_sort(ctx, tokens[:3], -1, order), lambda: B.sat_embed_bwd(ctx, order, out[:4], 1.0, gt),
                  lambda: B.sat_embed_bwd(ctx, order, out, 1.0, gt[:8]), lambda: B.sat_embed_bwd(ctx, order, out, 1.0, gt.half())):
        with pytest.raises(AssertionError):
            wrong()
    B.sat_sync_status(ctx)
