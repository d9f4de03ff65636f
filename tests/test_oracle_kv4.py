"""Pins of the oracle of the 4-bit node states (oracle/kv4.py)."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv4
from oracle.residual import bf16_to_f64, f64_to_bf16_rne


def _bf16(x):
    return bf16_to_f64(f64_to_bf16_rne(np.asarray(x, np.float64)))


def test_hand_worked_group():
    # least entry -2, largest 2: s = 4 / 16 = 1/4; cells [-2, -1.75), [-1.75, -1.5), ...; the largest entry's cell is held to 15
    x = np.full((1, 64), -2.0)
    x[0, :6] = [2.0, -1.75, -1.78125, 0.0, 0.25, -0.125]
    c, s, lo = kv4.encode(x)
    assert s[0, 0] == 0.25 and lo[0, 0] == -2.0
    assert c[0, :7].tolist() == [15, 1, 0, 8, 9, 7, 0]
    assert kv4.values(x)[0, :7].tolist() == [1.875, -1.625, -1.875, 0.125, 0.375, -0.125, -1.875]


def test_constant_group_is_exact_and_scale_is_rounded_to_nearest_even():
    x = np.concatenate([np.full(64, 3.25), np.full(64, -0.0)])[None]
    assert np.array_equal(kv4.values(x), x) and not kv4.encode(x)[1].any()
    # (hi - lo) / 16 = 257 / 256 lies half way between the bf16 numbers 1 and 1 + 2^-7: ties to even
    y = np.zeros((1, 64))
    y[0, 0], y[0, 1] = 16.0, -0.0625
    assert kv4.encode(y)[1][0, 0] == 1.0


def test_rounding_agrees_with_the_other_oracle_and_holds_for_subnormals():
    x = np.random.default_rng(1).standard_normal(500) * 10.0 ** np.random.default_rng(2).integers(-30, 30, 500)
    assert np.array_equal(kv4.round_to_bf16(x), _bf16(x))
    step = 2.0 ** -133
    assert kv4.round_to_bf16(np.array([0.5, 1.5, 2.5, -3.4, 0.0]) * step).tolist() == [0.0, 2 * step, 2 * step, -3 * step, 0.0]


@pytest.mark.parametrize("scale", [1e-30, 1.0, 1e30])
def test_codes_against_rational_arithmetic_and_the_error_bound(scale):
    rng = np.random.default_rng(3)
    x = _bf16(rng.standard_normal((5, 192)) * scale)
    c, s, lo = kv4.encode(x)
    v = kv4.values(x)
    for i in range(5):
        for j in range(192):
            f = (Fraction(x[i, j]) - Fraction(lo[i, j // 64])) / Fraction(s[i, j // 64])
            want = min(15, f.numerator // f.denominator)
            assert c[i, j] == want
            # half a cell, and where s was rounded down (by up to 2^-8 of itself) 16 such shortfalls at the top end
            assert abs(v[i, j] - x[i, j]) <= s[i, j // 64] * (0.5 + 16 * 2.0 ** -8)


def test_codes_next_to_a_border_are_those_of_the_exact_quotient():
    """Entries as little as 2^-130 from a whole number of cells above lo, which neither fp32 nor fp64 tells from the border."""
    tiny = 2.0 ** -np.arange(10.0, 131, 4)
    x = np.zeros((4, 64))
    x[:, 0], x[:, 1] = -4.0, 4.0
    x[0, 2:33], x[1, 2:33] = tiny, -tiny
    x[2, 0], x[2, 1], x[2, 2:33] = -2.0 ** -60, 4.0, 0.25 + 0 * tiny          # lo is what is tiny
    x[3, 0], x[3, 1], x[3, 2:33] = 2.0 ** -60, 4.0, 0.25 + 0 * tiny
    c, s, lo = kv4.encode(x)
    for i in range(4):
        for j in range(64):
            f = (Fraction(x[i, j]) - Fraction(lo[i, 0])) / Fraction(s[i, 0])
            assert c[i, j] == min(15, f.numerator // f.denominator), (i, j)
    assert c[0, 2:33].tolist() == [8] * 31 and c[1, 2:33].tolist() == [7] * 31
    assert c[2, 2] == 1 and c[3, 2] == 1          # (0, which the rest of the group is, is the least entry of the last)
