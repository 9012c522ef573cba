"""Microscaled matrices in numpy, from their definition and in 64 bits.  TEST INFRASTRUCTURE ONLY: nothing here is shared with, or
imported by, the CUDA library.

A row is cut into groups of 32 elements with one scale 2^e; an element is q 2^e with q in e4m3 (8 bits) or e2m1 (4 bits):
e = the least integer >= -127 with max |x| <= largest 2^e, q = x 2^-e rounded to nearest, ties to even.  A group with an
infinity or a NaN has the scale byte 255 and reads as NaN.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
LARGEST = {8: 448.0, 4: 6.0}


def magnitudes(bits: int) -> np.ndarray:
    """Non-negative numbers of the format by code."""
    mant, bias, count = (3, 7, 127) if bits == 8 else (1, 1, 8)
    c = np.arange(count)
    e, m = c >> mant, c & ((1 << mant) - 1)
    return np.where(e == 0, m / (1 << mant) * 2.0 ** (1 - bias), (1 + m / (1 << mant)) * 2.0 ** (e - bias))


def _least_exponent(amax: np.ndarray, bits: int) -> np.ndarray:
    e = np.full(amax.shape, -127, dtype=np.int64)
    pos = amax > 0
    guess = np.floor(np.log2(amax[pos] / LARGEST[bits])).astype(np.int64) - 1     # from below, whatever the logarithm's rounding
    for _ in range(4):
        guess = np.where(amax[pos] <= LARGEST[bits] * np.exp2(guess.astype(np.float64)), guess, guess + 1)
    e[pos] = np.maximum(guess, -127)
    return e


def row_bytes(d: int, bits: int) -> int:
    return (d + GROUP - 1) // GROUP * GROUP * bits // 8


def quantise(x: np.ndarray, bits: int):
    """(codes uint8 [rows, row_bytes], scales uint8 [rows, groups])"""
    rows, d = x.shape
    groups = (d + GROUP - 1) // GROUP
    full = np.zeros((rows, groups * GROUP), dtype=np.float64)
    full[:, :d] = x
    g = full.reshape(rows, groups, GROUP)
    bad = ~np.isfinite(g).all(axis=2)
    g = np.where(bad[:, :, None], 0.0, g)
    e = _least_exponent(np.abs(g).max(axis=2), bits)
    a = np.abs(g) * np.exp2(-e.astype(np.float64))[:, :, None]
    t = magnitudes(bits)
    mid = (t[:-1] + t[1:]) / 2                               # exact: a border between two neighbouring numbers
    up = np.searchsorted(mid, a, side="right")               # borders at or below a
    tie = (up > 0) & (mid[np.maximum(up - 1, 0)] == a) & (up % 2 == 1)
    code = (up - tie).astype(np.uint8)
    sign = np.signbit(g) & ~bad[:, :, None]
    code = (code | np.where(sign, 128 if bits == 8 else 8, 0).astype(np.uint8)).reshape(rows, groups * GROUP)
    if bits == 4:
        code = code[:, 0::2] | (code[:, 1::2] << 4)
    return code, np.where(bad, 255, e + 127).astype(np.uint8)


def dequantise(codes: np.ndarray, scales: np.ndarray, d: int, bits: int) -> np.ndarray:
    """fp64 [rows, d]"""
    c = codes.astype(np.int64)
    if bits == 4:
        c = np.stack([c & 15, c >> 4], axis=2).reshape(c.shape[0], -1)
    half = 128 if bits == 8 else 8
    t = np.append(magnitudes(bits), np.nan) if bits == 8 else magnitudes(bits)
    v = np.where(c >= half, -1.0, 1.0)[:, :d] * t[c % half][:, :d]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, GROUP, axis=1)[:, :d]
