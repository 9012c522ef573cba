"""Rows of fp32, bf16 and fp16 on the GPU for the tests of the row operators: matrices that lie inside a larger one, and what a rounding may be off."""
import numpy as np

U = 2.0 ** -24                                              # half a step of fp32
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}   # half of the least subnormal step
GUARD = -7.0


def dtype(t):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def matrix(a, t, extra=0):
    """a [rows, d] as the first columns of a larger matrix full of GUARD: (view, the larger one).  The row stride is a multiple of 16 bytes."""
    import torch
    a = np.asarray(a)
    rows, d = a.shape
    step = 4 if t == "f32" else 8
    full = torch.full((rows, (d + step - 1) // step * step + step * extra), GUARD, dtype=dtype(t), device="cuda")
    full[:, :d] = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda").to(dtype(t))
    return full[:, :d], full


def room(rows, d, t, extra=0):
    return matrix(np.full((rows, d), np.nan, dtype=np.float32), t, extra)


def guarded(full, d):
    """What lies behind the rows is as it was."""
    return bool((full[:, d:] == GUARD).all())


def host(t):
    return t.detach().double().cpu().numpy()


def rounding(want, t):
    """Off by rounding a number near `want` to the type once, to nearest."""
    return HALF[t] * np.abs(want) + LEAST[t]


def within(got, want, tol, what=""):
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / np.maximum(tol, 1e-300), 0)), bad.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} out of tolerance, worst at {i}: {got[i]!r} for {want[i]!r}, allowed {tol[i]:.3e}")
