"""Distillation of many classes where whole parts of a row are masked, where a row is far from zero, and where threads have no columns, at many temperatures.

Tolerances as in test_gpu_distill.py: a masked class adds nothing to a sum, and what a row's largest logit is does not count, only the distances from it.  A
logit of -inf stands in them as one that is 10,000 below.
"""
import numpy as np
import pytest

from oracle import rows_ref as ref
from tests.rows_util import U, guarded, host, matrix, room, within
from tests.test_gpu_distill import B, ctx, _dev, _tolerances   # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu
TEMPERATURES = [0.1, 1.0, 1.25, 2.0, 2.5, 5.0, 10.0, 20.0]
SHAPES = [(1100, 12), (1100, 200), (2000, 200), (4100, 64), (12000, 40), (20000, 64), (36000, 64), (70000, 30)]


def _check(B, ctx, z, ids, logits, T, hard, labels, t):
    import torch
    rows, classes = z.shape
    zt, _ = matrix(z, t, 1)
    g, full = room(rows, classes, t, 1)
    total, losses = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.full((rows,), np.nan, device="cuda")
    args = (_dev(ids, np.int32), _dev(logits), T, hard, _dev(labels, np.int32), None, 1.0 / rows)
    B.sat_distill_grad(ctx, zt, *args, total, g, losses)
    alone = torch.full((rows,), np.nan, device="cuda")
    B.sat_distill_grad(ctx, zt, *args, None, None, alone)
    B.sat_distill_grad(ctx, zt, *args, None, zt)
    zd = host(matrix(z, t)[0])
    B.sat_sync_status(ctx)
    w = np.full(rows, np.float32(1.0 / rows), dtype=np.float64)
    lg = np.asarray(logits, dtype=np.float32).astype(np.float64)
    h = float(np.float32(hard))
    want_l, want_g = ref.distill(zd, ids, lg, T, h, labels, w)
    near = np.where(np.isneginf(zd), np.max(zd, 1, keepdims=True) - 1e4, zd)
    tl, tg = _tolerances(near, ids, lg, T, h, labels, w, want_l, want_g, t)
    assert np.isfinite(want_l).all() and np.isfinite(tl).all() and np.isfinite(tg).all()
    what = f"T = {T}, {classes} classes, "
    within(host(losses), want_l, tl, what + "row losses")
    within(host(g), want_g, tg, what + "gradient")
    within(host(total), np.array([(w * want_l).sum()]), np.array([(w * (tl + 2 * U * np.abs(want_l))).sum() + 1e-12]), what + "loss")
    within(host(alone), want_l, tl, what + "row losses alone")
    assert guarded(full, classes) and torch.equal(g, zt)


def _masked(classes, t):
    """[patterns, classes]: parts of the row side by side, its beginning, its end, all columns of some threads, all but one class, all of it."""
    at = np.arange(classes)
    piece = at // (4 if t == "f32" else 8)
    return np.stack([(at >= classes // 3) & (at < 2 * classes // 3), at < classes // 2, at >= classes // 2, (piece % 128 >= 32) & (piece % 128 < 64), piece % 16 == 5, at != classes // 5,
                     np.ones(classes, dtype=bool)])


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hard", [0.0, 0.4])
@pytest.mark.parametrize("classes,k", SHAPES)
def test_masked_parts(B, ctx, classes, k, hard, t):
    rng = np.random.default_rng(classes + k)
    masks = [-6e4, -65504.0, -np.inf] if t == "f16" else [-np.inf, -3.3895e38 if t == "bf16" else np.finfo(np.float32).min, -1e30, -1e20, -1e10, -1e9]
    patterns = _masked(classes, t)
    rows = [(p, v) for p in patterns for v in masks if not (p.all() and v == -np.inf)]
    z, ids, logits, labels = 2 * rng.normal(size=(len(rows), classes)), np.full((len(rows), k), -1), 3 * rng.normal(size=(len(rows), k)), np.empty(len(rows), dtype=np.int64)
    for r, (p, v) in enumerate(rows):
        z[r, p] = v
        open_to = np.flatnonzero(~p) if not p.all() else np.arange(classes)     # what the teacher expects is not masked
        n = min(k, len(open_to))
        ids[r, :n] = rng.choice(open_to, n, replace=False)
        labels[r] = rng.choice(open_to)
    for T in TEMPERATURES:
        _check(B, ctx, z, ids, logits, T, hard, labels if hard else None, t)


@pytest.mark.parametrize("hard", [0.0, 0.4])
@pytest.mark.parametrize("classes,k", SHAPES)
def test_rows_far_from_zero(B, ctx, classes, k, hard):
    """Rows whose largest logit divided by T is near the number behind which a product with log2(e) / T keeps no fraction, and far behind it, to either side."""
    rng = np.random.default_rng(classes)
    sizes = [0.0, 1e3, 5e5, 7.2e5, 7.3e5, 1.5e6, 1e7, 2e9, 7e9, 1e12, 1e30]
    offsets = np.array([s * v for s in (1, -1) for v in sizes])[:, None]
    ids = np.stack([rng.choice(classes, k, replace=False) for _ in offsets])
    logits, labels = 3 * rng.normal(size=ids.shape), rng.integers(0, classes, len(ids))
    for T in (0.1, 1.0, 2.5, 10.0):
        z = offsets * T + rng.normal(size=(len(ids), classes)) * np.maximum(1.0, np.abs(offsets * T) * 2.0 ** -22)
        _check(B, ctx, z, ids, logits, T, hard, labels if hard else None, "f32")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("classes,k", [(1030, 129), (1100, 200), (1500, 256), (2000, 200), (2040, 130)])
def test_threads_without_columns(B, ctx, classes, k, t):
    rng = np.random.default_rng(classes)
    z, logits, labels = 2 * rng.normal(size=(9, classes)), 3 * rng.normal(size=(9, k)), rng.integers(0, classes, 9)
    ids = np.stack([rng.permutation(classes)[:k] for _ in z])
    for T in TEMPERATURES:
        for hard in (0.0, 0.4):
            _check(B, ctx, z, ids, logits, T, hard, labels if hard else None, t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.001, 0.02, 300.0, 1000.0])
@pytest.mark.parametrize("classes,k", [(60, 20), (1100, 200), (5003, 64), (20000, 64), (70000, 30)])
def test_the_ends_of_the_temperatures(B, ctx, classes, k, T, t):
    rng = np.random.default_rng(classes)
    z, logits, labels = 2 * rng.normal(size=(8, classes)), 3 * rng.normal(size=(8, k)), rng.integers(0, classes, 8)
    z[1] += 600.0                                                               # near, and behind, what a product with log2(e) / T takes at the lowest of them
    z[2] -= 900.0
    z[3] *= 1e4
    z[4:7, classes // 2:] = np.array([-np.inf, -1e5, -1e30])[:, None]
    ids = np.stack([rng.permutation(classes // 2)[:k] for _ in z])
    labels[4:7] = ids[4:7, 0]
    for hard in (0.0, 0.4):
        _check(B, ctx, z, ids, logits, T, hard, labels if hard else None, t)
