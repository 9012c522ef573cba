"""Distillation from a teacher's top logits, loss and gradient, against the definition in 64 bits.

Tolerances.  U = 2^-24 is fp32's half step.  An exponential of x / T, x = z - max, is off by 2^-22 (the instruction) and by 3 U |x| / T (two roundings of its
argument and one of x), relatively; a sum of C of them by the mean of that under the distribution and by the additions one after the other: C / 512 + 64 at
most.  A quotient adds 4 U.  The teacher's side is the same with k terms.  A logarithm of such a sum is off by its relative error and U of itself.
An exponential below 2^-126, the least normal number, is taken as zero (the largest of a row is 1): a gradient may lack 2^-126 of its factor.
"""
import numpy as np
import pytest

from oracle import rows_ref as ref
from tests.rows_util import HALF, U, guarded, host, matrix, room, rounding, within

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


def _dev(a, kind=np.float32):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=kind)).cuda()


def _inputs(rng, rows, classes, k, gaps=True):
    z = rng.normal(size=(rows, classes)) * np.exp(0.5 * rng.normal(size=(rows, 1))) * 2
    ids = np.stack([rng.permutation(classes)[:k] if classes < 5000 else rng.choice(classes, k, replace=False) for _ in range(rows)]).reshape(rows, k)
    logits = 3 * rng.normal(size=(rows, k))
    labels = rng.integers(0, classes, rows)
    if gaps and k:
        ids[::5, k // 2:] = -1
        ids[3::11] = -7
        logits[1::6, -1] = -np.inf
        ids[2::7, -1] = ids[2::7, 0]                                            # a class twice
        labels[::3] = ids[::3, 0]
        labels[4::9] = -1
    return z, ids, logits, labels


def _soft(v, T):
    x = (v - v.max()) / T
    e = np.exp(x)
    q = e / e.sum()
    return q, np.abs(x), np.log(e.sum())


def _tolerances(z, ids, logits, T, hard, labels, w, loss, g, t):
    rows, classes = z.shape
    tl, tg = np.zeros(rows), np.zeros((rows, classes))
    chain = (classes / 512 + 64) * U
    for r in range(rows):
        if w[r] == 0:
            continue
        ok = (ids[r] >= 0) & (ids[r] < classes) & ~np.isneginf(logits[r])
        if ok.any() and hard < 1:
            q, x, ls = _soft(z[r], T)
            p, y, lt = _soft(logits[r][ok], T)
            es, et = chain + 4 * U + (q * 3 * U * x).sum(), 80 * U + (p * 3 * U * y).sum()
            rq, rp = es + 8 * U + 3 * U * x, et + 8 * U + 3 * U * y
            at = ids[r][ok]
            gap = np.abs(y) + x[at]
            tl[r] += (1 - hard) * T * T * ((p * gap * (rp + 4 * U)).sum() + 70 * U * (p * gap).sum() + es + et + 4 * U * (abs(ls) + abs(lt)))
            add = q * rq
            np.add.at(add, at, p * (rp + 10 * U))
            tg[r] += abs(w[r]) * (1 - hard) * T * (add + 2.0 ** -126)
        if hard > 0 and labels is not None and 0 <= labels[r] < classes:
            q, x, ls = _soft(z[r], 1.0)
            es = chain + 4 * U + (q * 3 * U * x).sum()
            tl[r] += hard * (es + 4 * U * (abs(ls) + x[labels[r]]))
            add = q * (es + 8 * U + 3 * U * x)
            add[labels[r]] += 4 * U
            tg[r] += abs(w[r]) * hard * (add + 2.0 ** -126)
    return tl + 4 * U * np.abs(loss), tg + rounding(g, t) * 1.01 + 4 * U * np.abs(g)


def _run(B, ctx, z, ids, logits, T, hard, labels, rw, weight, t, extra=1):
    import torch
    rows, classes = z.shape
    zt, _ = matrix(z, t, extra)
    g, full = room(rows, classes, t, extra)
    total, losses = torch.full((1,), 0.75, dtype=torch.float64, device="cuda"), torch.full((rows,), np.nan, device="cuda")
    args = (_dev(ids, np.int32), _dev(logits), T, hard, _dev(labels, np.int32), _dev(rw), weight)
    B.sat_distill_grad(ctx, zt, *args, total, g, losses)
    B.sat_sync_status(ctx)
    assert guarded(full, classes)
    return zt, args, g, losses, total


def _check(B, ctx, z, ids, logits, T, hard, labels, rw, weight, t):
    import torch
    rows, classes = z.shape
    zt, args, g, losses, total = _run(B, ctx, z, ids, logits, T, hard, labels, rw, weight, t)
    w = np.full(rows, np.float32(weight), dtype=np.float64) * (1.0 if rw is None else rw.astype(np.float64))
    zd, lg = host(zt), np.asarray(logits, dtype=np.float32).astype(np.float64)
    want_l, want_g = ref.distill(zd, ids, lg, T, float(np.float32(hard)), labels, w)
    tl, tg = _tolerances(zd, ids, lg, T, hard, labels, w, want_l, want_g, t)
    within(host(losses), want_l, tl, "row losses")
    within(host(g), want_g, tg, "gradient")
    within(host(total), np.array([0.75 + (w * want_l).sum()]), np.array([(np.abs(w) * (tl + 2 * U * np.abs(want_l))).sum() + 1e-12]), "loss")
    only, again = torch.zeros(1, dtype=torch.float64, device="cuda"), room(rows, classes, t)[0]      # parts of it, and in place: the same bits
    B.sat_distill_grad(ctx, zt, *args, only)
    B.sat_distill_grad(ctx, zt, *args, None, again)
    B.sat_distill_grad(ctx, zt, *args, None, zt)
    B.sat_sync_status(ctx)
    assert torch.equal(again, g) and torch.equal(zt, g)
    within(host(only), host(total) - 0.75, np.array([1e-14 + 1e-14 * abs(float(total))]), "loss alone")


SHAPES = [(1, 1, 1), (5, 2, 2), (40, 7, 3), (33, 16, 16), (100, 41, 8), (50, 47, 20), (200, 64, 5), (64, 100, 33), (30, 121, 64), (21, 200, 200), (12, 256, 256), (10, 500, 40), (9, 1000, 100),
          (7, 1024, 256), (6, 1025, 12), (5, 5003, 64), (3, 32000, 256), (3, 50001, 64), (2, 131072, 30)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hard", [0.0, 0.4])
@pytest.mark.parametrize("rows,classes,k", SHAPES)
def test_loss_and_gradient(B, ctx, rows, classes, k, hard, t):
    rng = np.random.default_rng(rows + classes + k)
    z, ids, logits, labels = _inputs(rng, rows, classes, k)
    rw = np.exp(rng.normal(size=rows)).astype(np.float32)
    rw[::8] = 0.0
    T = [0.7, 1.0, 2.0, 4.0][(rows + classes) % 4]
    _check(B, ctx, z, ids, logits, T, hard, labels if hard else None, None if rows % 2 else rw, 64.0 / rows, t)


@pytest.mark.parametrize("classes", [5, 47, 300, 3000])
def test_labels_alone(B, ctx, classes):
    rng = np.random.default_rng(classes)
    z, ids, logits, labels = _inputs(rng, 37, classes, 4)
    _check(B, ctx, z, ids, logits, 1.5, 1.0, labels, None, 1 / 37, "f32")
    _check(B, ctx, z, ids[:, :0], logits[:, :0], 1.5, 0.5, labels, None, 1 / 37, "f32")
    _check(B, ctx, z, ids[:, :0], logits[:, :0], 1.5, 0.0, None, None, 1 / 37, "f32")     # nothing to learn from: zeros


@pytest.mark.parametrize("classes", [40, 700, 20000])
def test_many_rows_and_repeated_classes(B, ctx, classes):
    rng = np.random.default_rng(classes)
    rows, k = (3000, 30) if classes < 100 else (20, 90)
    z, _, logits, labels = _inputs(rng, rows, classes, k, gaps=False) if classes < 100 else _inputs(rng, rows, classes, k, gaps=False)
    ids = rng.integers(0, min(classes, 12), (rows, k))                          # every class several times
    _check(B, ctx, z, ids, logits, 2.0, 0.3, labels, None, 1.0 / rows, "f32")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [9, 47, 600, 4000])
def test_rows_that_are_no_numbers(B, ctx, classes, t):
    """They reach their own row and nothing else, and not even that where its weight is 0."""
    rng = np.random.default_rng(classes)
    z, ids, logits, labels = _inputs(rng, 24, classes, 6, gaps=False)
    z[1, 3], z[2, :], z[3, 5] = np.nan, -np.inf, np.inf
    z[4, classes - 1] = -np.inf                                                 # a class of probability 0
    ids[4, ids[4] == classes - 1] = 0
    labels[4] = 1
    z[5] = np.finfo(np.float32).min if t == "f32" else -3e38
    z[5, ids[5, 0]] = 3.0
    logits[6, 2], logits[7, 1] = np.nan, np.inf
    logits[8] = -np.inf
    z[9:12] = z[1:4]
    rw = np.ones(24, dtype=np.float32)
    rw[9:12] = 0.0
    ids[12, 0] = classes - 1
    z[12, classes - 1] = -np.inf                                                # ... that the teacher expects
    labels[12] = 0
    zt, args, g, losses, total = _run(B, ctx, z, ids, logits, 2.0, 0.25, labels, rw, 1.0, t)
    got, loss = host(g), host(losses)
    for r in (1, 2, 3, 6, 7):
        assert np.isnan(loss[r]) and np.isnan(got[r]).any()
    assert np.all(got[9:12] == 0) and np.all(loss[9:12] == 0)
    assert loss[12] == np.inf and np.isfinite(got[12]).all()
    rest = np.array([r for r in range(24) if r not in (1, 2, 3, 5, 6, 7, 9, 10, 11, 12)])
    want_l, want_g = ref.distill(host(zt)[rest], ids[rest], logits[rest].astype(np.float32), 2.0, 0.25, labels[rest], rw[rest])
    finite = np.where(np.isneginf(host(zt)[rest]), -1e4, host(zt)[rest])
    tl, tg = _tolerances(finite, ids[rest], logits[rest].astype(np.float32).astype(np.float64), 2.0, 0.25, labels[rest], rw[rest], want_l, want_g, t)
    within(loss[rest], want_l, tl, "row losses")
    within(got[rest], want_g, tg, "gradient")
    # an exact gradient adds up to zero; each of these is rounded to its type
    assert np.isfinite(got[5]).all() and abs(got[5].sum()) < 1e-5 + HALF[t] * np.abs(got[5]).sum()


@pytest.mark.parametrize("classes", [47, 3000])
def test_ids_and_labels_outside(B, ctx, classes):
    import torch
    rng = np.random.default_rng(classes)
    z, ids, logits, labels = _inputs(rng, 30, classes, 5)
    ids[0, 1], labels[7], ids[20, 4] = classes, classes + 3, 2 ** 31 - 1
    zt, _ = matrix(z, "f32")
    g, losses = room(30, classes, "f32")[0], torch.empty(30, device="cuda")
    B.sat_distill_grad(ctx, zt, _dev(ids, np.int32), _dev(logits), 1.0, 0.5, _dev(labels, np.int32), None, 1.0, None, g, losses)
    with pytest.raises(B.SatError) as e:
        B.sat_sync_status(ctx)
    assert e.value.status == B.SAT_EDATA
    B.sat_sync_status(ctx)
    want_l, want_g = ref.distill(host(zt), ids, logits.astype(np.float32), 1.0, 0.5, labels, np.ones(30))
    tl, tg = _tolerances(host(zt), ids, logits.astype(np.float32).astype(np.float64), 1.0, 0.5, labels, np.ones(30), want_l, want_g, "f32")
    within(host(losses), want_l, tl, "row losses")
    within(host(g), want_g, tg, "gradient")


def test_gradient_is_a_difference(B, ctx):
    """The kernel's own losses at moved logits: (loss(z + h e_c) - loss(z - h e_c)) / 2h.  A loss of about 1 is off by 2^-22 or so, over 2h = 2^-5; the third
    derivative, at most 1, leaves h^2 / 6."""
    import torch
    rng = np.random.default_rng(5)
    classes, h = 24, 2.0 ** -6
    z, ids, logits, labels = _inputs(rng, 1, classes, 5, gaps=False)
    z = np.clip(z, -2, 2)
    moved = np.concatenate([z, np.repeat(z, 2 * classes, 0)]).astype(np.float32)
    for c in range(classes):
        moved[1 + c, c] += h
        moved[1 + classes + c, c] -= h
    n = len(moved)
    rep = lambda a: np.repeat(a, n, 0)
    _, _, g, losses, _ = _run(B, ctx, moved, rep(ids), rep(logits), 1.5, 0.3, rep(labels), None, 1.0, "f32")
    loss = host(losses)
    step = moved[1:1 + classes].astype(np.float64)[np.arange(classes), np.arange(classes)] - moved[1 + classes:].astype(np.float64)[np.arange(classes), np.arange(classes)]
    diff = (loss[1:1 + classes] - loss[1 + classes:]) / step
    tl, _ = _tolerances(moved[:1].astype(np.float64), ids, logits, 1.5, 0.3, labels, np.ones(1), loss[:1], host(g)[:1], "f32")
    assert np.all(np.abs(diff - host(g)[0]) <= 2 * tl[0] / (2 * h) * 1.5 + h * h / 6 + 1e-6)


def test_no_rows(B, ctx):
    import torch
    total = torch.full((1,), 2.0, dtype=torch.float64, device="cuda")
    z, ids, logits = torch.empty((0, 8), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty((0, 3), device="cuda")
    B.sat_distill_grad(ctx, z, ids, logits, 1.0, 0.0, None, None, 1.0, total, z)
    B.sat_sync_status(ctx)
    assert float(total) == 2.0


def test_offsets_beyond_32_bits(B, ctx):
    import torch
    rows, classes, ld = 70000, 12, 32768
    big = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")
    z = big[:, :classes]
    z.normal_()
    near = torch.empty((rows, 16), dtype=torch.bfloat16, device="cuda")[:, :classes]
    near.copy_(z)
    ids, logits = torch.randint(0, classes, (rows, 3), device="cuda", dtype=torch.int32), torch.randn(rows, 3, device="cuda")
    B.sat_distill_grad(ctx, near, ids, logits, 2.0, 0.0, None, None, 1.0, None, near)
    B.sat_distill_grad(ctx, z, ids, logits, 2.0, 0.0, None, None, 1.0, None, z)
    B.sat_sync_status(ctx)
    assert torch.equal(z, near)


def test_on_a_side_stream_and_in_a_graph(B):
    import torch
    stream = torch.cuda.Stream()
    ctx = B.sat_create(0, stream.cuda_stream)
    try:
        for classes in (47, 6000):
            z, z2, g, want = (torch.randn(50, classes + (-classes) % 4, device="cuda")[:, :classes] for _ in range(4))
            ids, logits = torch.randint(0, classes, (50, 9), device="cuda", dtype=torch.int32), torch.randn(50, 9, device="cuda")
            total, want_total = (torch.zeros(1, dtype=torch.float64, device="cuda") for _ in range(2))
            torch.cuda.synchronize()
            call = lambda zz, gg, tt: B.sat_distill_grad(ctx, zz, ids, logits, 2.0, 0.0, None, None, 0.02, tt, gg)
            with torch.cuda.stream(stream):
                call(z2, want, want_total)
                stream.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    call(z, g, total)
                z.copy_(z2)
                total.zero_()
                graph.replay()
                graph.replay()
                stream.synchronize()
            assert torch.equal(g, want) and abs(float(total) - 2 * float(want_total)) < 1e-12
            del graph
    finally:
        B.sat_destroy(ctx)


def test_refusals(B, ctx):
    import torch
    z, g, ids, logits, labels = torch.zeros(4, 8, device="cuda"), torch.full((4, 8), 3.0, device="cuda"), _dev(np.zeros((4, 2)), np.int32), torch.zeros(4, 2, device="cuda"), _dev(np.zeros(4), np.int32)
    p, lib, nan = (lambda t: t.data_ptr()), B._lib, float("nan")
    before = B.sat_launch_count(ctx)
    F = lambda n=4, c=8, t=0, z=p(z), ld=8, k=2, i=p(ids), l=p(logits), T=1.0, h=0.5, y=p(labels), s=None, rl=None, g=p(g), ldg=8: lib.sat_distill_grad(ctx, n, c, t, z, ld, k, i, l, T, h, y, None, 1.0, s, rl, g, ldg)
    for bad in (F(n=-1), F(n=2 ** 31), F(c=0), F(c=9), F(c=2 ** 31 - 1), F(t=4), F(z=None), F(z=p(z) + 4), F(ld=10), F(k=-1), F(k=257), F(i=None), F(l=None), F(T=0.0), F(T=-1.0), F(T=nan), F(T=1e4),
                F(T=1e-4), F(h=-0.1), F(h=1.1), F(h=nan), F(y=None), F(g=None), F(g=p(g) + 8), F(ldg=6), F(t=1, ld=12)):
        assert bad == B.SAT_EINVAL
    assert B.sat_launch_count(ctx) == before and bool((g == 3).all())
    call = lambda **kw: B.sat_distill_grad(ctx, kw.get("z", z), kw.get("ids", ids), kw.get("logits", logits), 1.0, 0.5, kw.get("labels", labels), kw.get("rw"), 1.0, kw.get("s"), kw.get("g", g))
    for kw in (dict(z=z.double()), dict(ids=ids.long()), dict(ids=ids[:3]), dict(logits=logits.half()), dict(logits=logits[:, :1]), dict(labels=labels[:3]), dict(rw=labels), dict(g=g[:3]),
               dict(g=g.half()), dict(s=torch.zeros(1, device="cuda"))):
        with pytest.raises(AssertionError):
            call(**kw)
    B.sat_sync_status(ctx)
