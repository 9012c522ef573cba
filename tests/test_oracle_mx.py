"""The 64-bit reference of the microscaled formats (oracle/mx_ref.py) against published tables, brute force and worked examples."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import mx_ref as mx


def test_every_number_of_the_formats():
    import torch
    got = mx.magnitudes(8)
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, want)
    assert np.array_equal(mx.magnitudes(4), [0, 0.5, 1, 1.5, 2, 3, 4, 6])


@pytest.mark.parametrize("bits", [8, 4])
def test_elements_are_the_nearest_numbers_with_ties_to_even(bits):
    rng = np.random.default_rng(bits)
    t = mx.magnitudes(bits)
    mids = (t[1:] + t[:-1]) / 2
    probe = np.concatenate([t, mids, np.nextafter(mids, 0), np.nextafter(mids, 1e9), rng.uniform(0, t[-1], 200)])
    for v in probe:
        x = np.zeros((1, 32), dtype=np.float64)
        x[0, 0], x[0, 1], x[0, 2] = t[-1], v, -v              # the largest number fixes the scale at one
        code, scale = mx.quantise(x, bits)
        assert scale[0, 0] == 127
        dist = [abs(Fraction(float(v)) - Fraction(float(n))) for n in t]
        near = [i for i, d in enumerate(dist) if d == min(dist)]
        want = near[0] if len(near) == 1 else [i for i in near if i % 2 == 0][0]
        got = int(code[0, 1]) if bits == 8 else int(code[0, 0] >> 4)
        assert got == want, (v, got, want)
        neg = int(code[0, 2]) if bits == 8 else int(code[0, 1] & 15)
        assert neg == want + (128 if bits == 8 else 8)


@pytest.mark.parametrize("bits,amax,e", [
    (8, 448.0, 0), (8, np.nextafter(np.float32(448), np.float32(1e9)), 1), (8, 224.0, -1), (8, 1.0, -8), (8, 1.75, -8), (8, 1.76, -7),
    (8, 2.0 ** -119, -127), (8, 2.0 ** -149, -127), (8, 0.0, -127), (8, np.finfo(np.float32).max, 120),
    (4, 6.0, 0), (4, np.nextafter(np.float32(6), np.float32(1e9)), 1), (4, 3.0, -1), (4, 1.0, -2), (4, 1.5, -2), (4, 1.51, -1),
    (4, 2.0 ** -126, -127), (4, 0.0, -127), (4, np.finfo(np.float32).max, 126)])
def test_the_scale_is_the_least_that_fits(bits, amax, e):
    x = np.zeros((1, 5), dtype=np.float32)
    x[0, 3] = -amax
    _, scale = mx.quantise(x, bits)
    assert int(scale[0, 0]) == e + 127


@pytest.mark.parametrize("bits", [8, 4])
def test_round_trip_error_and_fixed_point(bits):
    rng = np.random.default_rng(3)
    x = (rng.normal(size=(40, 71)) * np.exp(3 * rng.normal(size=(40, 71)))).astype(np.float32)
    c, s = mx.quantise(x, bits)
    assert c.shape == (40, mx.row_bytes(71, bits)) and s.shape == (40, 3)
    y = mx.dequantise(c, s, 71, bits)
    scale = np.repeat(np.exp2(s.astype(np.float64) - 127), 32, axis=1)[:, :71]
    half, least = (2.0 ** -4, 2.0 ** -10) if bits == 8 else (0.25, 0.25)
    assert np.all(np.abs(y - x) <= np.maximum(half * np.abs(x), least * scale))
    c2, s2 = mx.quantise(y, bits)                              # scales may shrink where the largest element was rounded down a binade
    assert np.array_equal(mx.dequantise(c2, s2, 71, bits), y)


def test_worked_example_and_what_is_not_finite():
    x = np.zeros((2, 34), dtype=np.float32)
    x[0, :4] = [12.0, -5.0, 0.49, 3.5]                         # 4 bits: scale 2; 6, -2.5 -> -2, .245 -> 0, 1.75 -> 2
    x[0, 33] = 0.75                                            # a group of two elements: scale 1/8, code of 6
    x[1, 5], x[1, 33] = np.inf, 1.0
    c, s = mx.quantise(x, 4)
    assert list(s[0]) == [128, 124] and list(c[0, :2]) == [7 | (4 | 8) << 4, 0 | 4 << 4] and c[0, 16] == 7 << 4 and not c[0, 17:].any()
    assert list(s[1]) == [255, 125] and not c[1, :16].any()
    y = mx.dequantise(c, s, 34, 4)
    assert np.isnan(y[1, :32]).all() and y[1, 33] == 1.0 and list(y[0, :4]) == [12.0, -4.0, 0.0, 4.0]
