"""Angles of large frequencies: the fraction of a turn is right to 64 bits, so that an
angle is off by at most 2e-7 radians at any position, whatever the finite frequency."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la


def _arctan_of_inverse(n, digits):
    """arctan(1 / n) 10^digits, by its series."""
    one, total, k, sign = 10 ** digits // n, 0, 1, 1
    while one:
        total += sign * (one // k)
        one //= n * n
        k, sign = k + 2, -sign
    return total


def _two_pi(digits):
    """Machin: pi = 16 arctan(1/5) - 4 arctan(1/239)."""
    more = digits + 20
    return Fraction(2 * (16 * _arctan_of_inverse(5, more) - 4 * _arctan_of_inverse(239, more)), 10 ** more)


TWO_PI = _two_pi(400)                            # the largest double has 309 digits
FREQ = [1.0, 3.14159, 3.1416, np.pi, 2 * np.pi, 6.3, 12.566, 100.25, -7.0, 12345.678, 54321.9, -54321.9, 1e6, 2.0 ** 40 + 0.5, 1e15,
        1e19, 1e22, -1e22, 1e100, -1e300, 1.7976931348623157e308]


def _turns(f):
    x = Fraction(float(f)) / TWO_PI
    return x - (x.numerator // x.denominator)


def _from_half(x):
    """The distance to the nearest whole turn."""
    x = abs(x) % 1
    return min(x, 1 - x)


def test_large_frequencies_have_64_bits_of_a_turn():
    """With long doubles of 64 bits: a sine and a cosine off by a unit of their last each move an
    angle by 2^-63, the arctangent's unit is 2^-62 (up to pi): 3 2^-63 / 2 pi = 0.95 2^-64 of a turn.
    The quotient's and the divisor's rounding, 0.75 of that, a whole turn more, 0.5, and what is cut off, 1."""
    for f, t in zip(FREQ, la.la_rope_turns(FREQ)):
        assert _from_half(_turns(f) - Fraction(int(t), 2 ** 64)) <= Fraction(4, 2 ** 64), f


def test_bases_below_one():
    """The frequencies that these give are large."""
    freq = la.la_rope_frequencies(64, 1e-6)
    assert freq.max() > 1e5
    for f, t in zip(freq, la.la_rope_turns(freq)):
        assert _from_half(_turns(f) - Fraction(int(t), 2 ** 64)) <= Fraction(4, 2 ** 64), f


@pytest.mark.gpu
def test_far_positions_at_large_frequencies():
    """(1, 0) turned is the angle's cosine and sine, off by at most 2.7e-7 (the angle by 2e-7 at
    most, the polynomials by 2e-9, two roundings) and half an ulp."""
    pos = [1, 5, 131071, 1000003, 2 ** 30 + 1, 2 ** 31 - 1, -1, -2 ** 31]
    n = 2 * len(FREQ)
    dim = -(-n // 8) * 8
    rope = api.Rope(dim, n, "pairs", frequencies=np.array(FREQ))
    x = torch.zeros((len(pos), 1, dim), device="cuda")
    x[:, :, 0:n:2] = 1.0
    y = torch.empty_like(x)
    rope.apply(x, None, y, positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    y = y.double().cpu().numpy()[:, 0]
    for i, f in enumerate(FREQ):
        for t, p in enumerate(pos):
            a = Fraction(float(f)) * p / TWO_PI
            a = 2 * np.pi * float(a - round(a))
            off = max(abs(y[t, 2 * i] - np.cos(a)), abs(y[t, 2 * i + 1] - np.sin(a)))
            assert off <= 2.7e-7 + 2.0 ** -24, (f, p, off)
