"""Row losses of distillation at high temperatures and of students that all but agree with their teacher, against the definition in 64 bits.

T^2 KL is of the order of the logits' own differences at any T, and its tolerance here is relative to it.  With p and q the teacher's and the student's
probabilities, D_j = t_j - z_j and u_j = (D_j - sum p D) / T,  KL = log(1 + A + R),  A = sum p (e^-u - 1 + u),  R what the classes that the teacher does not name add.

Up to KL = 1/8 the kernel (1,024 classes at most, T above 4) works that out.  U = 2^-24.  A difference D is off by 2 U (|t - max t| + |z - max z|), the mean by the
mean of that and by additions (80 U of the mean magnitude); A moves by sum p |1 - e^-u| times that over T, and by 200 U and 3 U max |t - max t| / T of itself (exponentials, their
sums, products).  R is off by 200 U of itself, by 3 U of the mean |z - max z| / T in it, and by what the mean is off.  The logarithm and the factors add 8 U.
Above 1/8 the tolerance is that of test_gpu_distill.py.  Between the two sides of 1/8 (1e-3 of it) either holds.
"""
import numpy as np
import pytest

from oracle import rows_ref as ref
from tests.rows_util import U, host, matrix, room, within
from tests.test_gpu_distill import B, ctx, _dev, _tolerances   # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


def _near(z, ids, logits, T):
    """Of a row without a class named twice: (KL, what T^2 times it may be off over T^2)"""
    ok = (ids >= 0) & ~np.isneginf(logits)
    t, at = logits[ok], ids[ok]
    g, x = t - t.max(), z - z.max()
    w = np.exp(g / T)
    p = w / w.sum()
    D = g - x[at]
    mean = (p * D).sum()
    u = (D - mean) / T
    rest = np.ones(len(z), dtype=bool)
    rest[at] = False
    e = np.exp(x / T) * rest
    R = np.exp(mean / T) * e.sum() / w.sum()
    A = (p * np.where(np.abs(u) < 1e-2, u * u * (0.5 - u / 6 + u * u / 24 - u ** 3 / 120 + u ** 4 / 720), np.expm1(-u) + u)).sum()
    each = 2 * U * (np.abs(g) + np.abs(x[at]))
    centre = (p * each).sum() + 80 * U * (p * np.abs(D)).sum()
    tol = (p * np.abs(np.expm1(-u)) * (each + 2 * U * np.abs(D - mean) + centre)).sum() / T + A * (200 * U + 3 * U * np.abs(g).max() / T)
    tol += R * (200 * U + (centre + 2 * U * abs(mean)) / T) + 3 * U * np.exp(mean / T) * (e * np.where(rest, np.abs(x), 0) / T)[e > 0].sum() / w.sum()
    return np.log1p(A + R), tol + 8 * U * (A + R)


def _check(B, ctx, z, ids, logits, T, hard, labels, t, sharp):
    import torch
    rows, classes = z.shape
    zt, _ = matrix(z, t, 1)
    g = room(rows, classes, t, 1)[0]
    new = lambda: torch.full((rows,), np.nan, device="cuda")
    losses, alone, placed, total = new(), new(), new(), torch.zeros(1, dtype=torch.float64, device="cuda")
    args = (_dev(ids, np.int32), _dev(logits), T, hard, _dev(labels, np.int32), None, 1.0)
    zd = host(zt)
    B.sat_distill_grad(ctx, zt, *args, total, g, losses)
    B.sat_distill_grad(ctx, zt, *args, None, None, alone)
    B.sat_distill_grad(ctx, zt, *args, None, zt, placed)
    B.sat_sync_status(ctx)
    assert torch.equal(losses, alone) and torch.equal(losses, placed) and torch.equal(g, zt)
    lg, h = np.asarray(logits, dtype=np.float32).astype(np.float64), float(np.float32(hard))
    want, want_g = ref.distill(zd, ids, lg, T, h, labels, np.ones(rows))
    far, tg = _tolerances(zd, ids, lg, T, h, labels, np.ones(rows), want, want_g, t)
    tol = far.copy()
    for r in range(rows):
        kl, near = _near(zd[r], ids[r], lg[r], T)
        if kl < 0.125 * 1.001:
            label, _ = _tolerances(zd[r:r + 1], ids[r:r + 1] * 0 - 1, lg[r:r + 1], T, h, None if labels is None else labels[r:r + 1], np.ones(1), want[r:r + 1] * 0, want_g[r:r + 1], t)
            near = (1 - h) * T * T * near + label[0] + 4 * U * want[r]
            tol[r] = near if kl < 0.125 * 0.999 else max(near, far[r])
            want[r] = (1 - h) * T * T * kl + (want[r] - (1 - h) * _plain(zd[r], ids[r], lg[r], T))   # (the definition itself cancels in 64 bits as well)
    assert hard > 0 or tol.sum() <= sharp * want.sum()                          # the tolerance says something (of all rows: two classes may be alike by chance)
    within(host(losses), want, tol, f"T = {T}, {classes} classes, row losses")
    within(host(g), want_g, tg, f"T = {T}, {classes} classes, gradient")
    within(host(total), np.array([host(losses).sum()]), np.array([1e-13 * np.abs(host(losses)).sum()]), "loss")


def _plain(z, ids, logits, T):
    return ref.distill(z[None], ids[None], logits[None], T, 0.0, None, np.ones(1))[0][0]


def _students(rng, rows, classes, k, kind):
    """Logits of students and teachers: unlike each other, alike up to 1e-3, and alike up to 0.3; the classes that the teacher does not name are not likely"""
    ids = np.stack([rng.permutation(classes)[:k] for _ in range(rows)])
    logits = (2 * rng.normal(size=(rows, k))).astype(np.float32).astype(np.float64)
    z = 2 * rng.normal(size=(rows, classes)) - (0 if kind == "other" else 12)
    if kind != "other":
        np.put_along_axis(z, ids, logits + {"alike": 1e-3, "similar": 0.3}[kind] * rng.normal(size=(rows, k)), 1)
        z += rng.normal(size=(rows, 1))
    return z, ids, logits, rng.integers(0, classes, rows)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["other", "alike", "similar"])
@pytest.mark.parametrize("classes,k", [(2, 2), (3, 3), (7, 7), (16, 16), (47, 47), (64, 64), (65, 65), (130, 130), (200, 200), (256, 256), (47, 8), (100, 99), (300, 256), (520, 256), (1000, 256), (1024, 200)])
def test_high_temperatures(B, ctx, classes, k, kind, t):
    rng = np.random.default_rng(classes + k)
    z, ids, logits, labels = _students(rng, 37, classes, k, kind)
    for T in (4.5, 20.0, 100.0, 1000.0):
        for hard in (0.0, 0.3):
            _check(B, ctx, z, ids, logits, T, hard, labels if hard else None, t, 1e-3 if kind != "alike" else 3e-2)


@pytest.mark.parametrize("classes,k", [(7, 7), (47, 40), (200, 150), (1000, 256)])
def test_missing_entries_and_masked_classes(B, ctx, classes, k):
    rng = np.random.default_rng(classes)
    z, ids, logits, _ = _students(rng, 37, classes, k, "similar")
    ids[::5, k // 2:] = -1
    logits[1::5, -1] = -np.inf
    for r in range(2, 37, 5):                                                   # classes that the teacher does not name cannot be had, or hardly
        off = np.setdiff1d(np.arange(classes), ids[r])
        z[r, off] = [-1e9, -1e30, -3e38][r % 3]
    for T in (4.5, 20.0, 1000.0):
        _check(B, ctx, z, ids, logits, T, 0.0, None, "f32", 1e-3)


@pytest.mark.parametrize("classes,k", [(5, 9), (47, 30), (300, 200)])
def test_classes_named_twice(B, ctx, classes, k):
    """Their losses are not those of a sum without cancellation: as at low temperatures."""
    import torch
    rng = np.random.default_rng(classes)
    ids, logits = rng.integers(0, classes, (40, k)), rng.normal(size=(40, k))
    z = rng.normal(size=(40, classes))
    for T in (5.0, 50.0):
        zt, g, losses = matrix(z, "f32")[0], room(40, classes, "f32")[0], torch.empty(40, device="cuda")
        B.sat_distill_grad(ctx, zt, _dev(ids, np.int32), _dev(logits), T, 0.0, None, None, 1.0, None, g, losses)
        B.sat_sync_status(ctx)
        lg = logits.astype(np.float32).astype(np.float64)
        want, want_g = ref.distill(host(zt), ids, lg, T, 0.0, None, np.ones(40))
        tl, tg = _tolerances(host(zt), ids, lg, T, 0.0, None, np.ones(40), want, want_g, "f32")
        within(host(losses), want, tl, "row losses")
        within(host(g), want_g, tg, "gradient")


def test_rows_that_are_no_numbers(B, ctx):
    """They reach their own row and nothing else, beside rows that agree with their teacher."""
    import torch
    rng = np.random.default_rng(2)
    z, ids, logits, _ = _students(rng, 40, 30, 30, "alike")
    z[3, 4], z[9, :], z[15, 2], logits[21, 5], logits[22, 6] = np.nan, -np.inf, np.inf, np.nan, np.inf
    rw = np.ones(40, dtype=np.float32)
    rw[25] = 0.0
    z[25] = np.nan
    bad = np.zeros(40, dtype=bool)
    bad[[3, 9, 15, 21, 22]] = True
    zt, g, losses = matrix(z, "f32")[0], room(40, 30, "f32")[0], torch.empty(40, device="cuda")
    B.sat_distill_grad(ctx, zt, _dev(ids, np.int32), _dev(logits), 20.0, 0.0, None, _dev(rw), 1.0, None, g, losses)
    B.sat_sync_status(ctx)
    assert np.isnan(host(losses)[bad]).all() and np.isnan(host(g)[bad]).any(1).all()
    assert host(losses)[25] == 0 and bool((g[25] == 0).all())
    for r in np.flatnonzero(~bad & (np.arange(40) != 25)):
        kl, tol = _near(host(zt)[r], ids[r], logits[r].astype(np.float32).astype(np.float64), 20.0)
        assert abs(host(losses)[r] - 400 * kl) <= 400 * tol + 4 * U * 400 * kl


@pytest.mark.parametrize("classes,k", [(7, 5), (47, 8), (47, 30), (200, 40), (900, 200), (1500, 30)])
@pytest.mark.parametrize("T", [4.0, 5.0])
def test_the_gradient_does_not_depend_on_what_else_is_asked_for(B, ctx, classes, k, T):
    import torch
    rng = np.random.default_rng(classes)
    z, ids, logits, labels = _students(rng, 50, classes, k, "similar")
    zt, (g, alone) = matrix(z, "f32")[0], (room(50, classes, "f32")[0] for _ in range(2))
    args = (_dev(ids, np.int32), _dev(logits), T, 0.5, _dev(labels, np.int32), None, 0.02)
    B.sat_distill_grad(ctx, zt, *args, torch.zeros(1, dtype=torch.float64, device="cuda"), g, torch.empty(50, device="cuda"))
    B.sat_distill_grad(ctx, zt, *args, None, alone)
    B.sat_sync_status(ctx)
    assert torch.equal(g, alone)
