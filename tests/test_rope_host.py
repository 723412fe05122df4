"""Rotary positions on the CPU: frequencies, turns, and what the entry points and
the binding refuse before any launch (device pointers are dummies)."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import rope as orope
from paper_2609_15030_amd import linattn as la

P = 0x10000
LIB = la.library()


@pytest.mark.parametrize("rotary", [2, 4, 10, 64, 128, 512])
@pytest.mark.parametrize("scaling", [None, ("linear", 4.0), ("base", 8.0), ("parts", 4.0, 4096.0, 1.0, 32.0)], ids=str)
def test_frequencies(rotary, scaling):
    got = la.la_rope_frequencies(rotary, 1e4, None if scaling is None else la.make_rope_scaling(*scaling))
    want = orope.frequencies(rotary, 1e4, *(scaling or ()))
    # each is a power, a quotient and a few sums in fp64; the power's error grows with its exponent's size (log 1e4 < 10)
    assert np.allclose(got, want, rtol=40 * 2.0 ** -53, atol=0)


def test_turns_are_fractions_of_a_turn():
    """Off by less than a unit of 2^-64 and the fp64 quotient's 2^-63 of the turns."""
    freq = np.array([0.0, 1.0, 1e-4, math.pi, 2 * math.pi, 12345.678, -0.25, 1e-30])
    turns = la.la_rope_turns(freq)
    two_pi = Fraction(6283185307179586476925286766559005768394, 10 ** 39)
    for f, t in zip(freq, turns):
        x = Fraction(float(f)) / two_pi
        off = (x - (x.numerator // x.denominator)) - Fraction(int(t), 2 ** 64)
        off -= round(off)                                        # just below a whole turn may be none
        assert abs(off) <= Fraction(1, 2 ** 63) * (1 + abs(x))


@pytest.mark.parametrize("args", [(0, 1e4), (-2, 1e4), (7, 1e4), (514, 1e4), (64, 0.0), (64, -1.0), (64, float("nan")),
                                  (64, float("inf"))])
def test_frequencies_are_refused(args):
    with pytest.raises(la.LinAttnError):
        la.la_rope_frequencies(*args)


@pytest.mark.parametrize("scaling", [("linear", 0.0), ("base", -1.0), ("linear", float("nan")), ("parts", 4.0),
                                     ("parts", 4.0, 4096.0, 32.0, 1.0), ("parts", 4.0, 4096.0, 1.0, 1.0),
                                     ("parts", 4.0, -1.0, 1.0, 32.0), ("parts", float("inf"), 4096.0, 1.0, 32.0),
                                     ("parts", 4.0, 4096.0, float("nan"), 32.0)], ids=str)
def test_scalings_are_refused(scaling):
    with pytest.raises(la.LinAttnError):
        la.la_rope_frequencies(64, 1e4, la.make_rope_scaling(*scaling))


def test_other_host_calls_are_refused():
    with pytest.raises(ValueError):
        la.make_rope_scaling("quadratic", 2.0)
    with pytest.raises(la.LinAttnError):
        la.la_rope_turns([1.0, float("inf")])
    with pytest.raises(la.LinAttnError):
        la.la_rope_turns(np.zeros(0))
    with pytest.raises(la.LinAttnError):
        la.la_rope_turns(np.zeros(257))
    assert LIB.la_rope_frequencies(64, 1e4, None, None) == la.LA_ERR_INVALID_ARG
    bad = la.LaRopeScaling(9, 1.0, 1.0, 0.0, 1.0)
    assert LIB.la_rope_frequencies(64, 1e4, ctypes.byref(bad), P) == la.LA_ERR_INVALID_ARG
    assert LIB.la_rope_turns(None, 4, P) == la.LA_ERR_INVALID_ARG


def _apply(plan=None, q=None, k=None, n=5, at=None, **kw):
    p = plan or la.LaRopePlan(128, 128, la.LA_ROPE_HALVES, la.LA_BF16, 1.0, P)
    for name, v in kw.items():
        setattr(p, name, v)
    at = la.LaRopePositions(P, None, 0, None) if at is None else at
    by = lambda x: None if x is None else ctypes.byref(x)
    return LIB.la_rope_apply(by(p), by(q or la.LaRopeRows(P, P + 4096, 4, 0, 0)), by(k), n, by(at), 0, None)


@pytest.mark.parametrize("change,want", [
    (dict(head_dim=0), la.LA_ERR_UNSUPPORTED), (dict(head_dim=100), la.LA_ERR_UNSUPPORTED),
    (dict(rotary_dim=0), la.LA_ERR_INVALID_ARG), (dict(rotary_dim=63), la.LA_ERR_INVALID_ARG),
    (dict(rotary_dim=130), la.LA_ERR_INVALID_ARG), (dict(head_dim=1024, rotary_dim=514), la.LA_ERR_UNSUPPORTED),
    (dict(layout=2), la.LA_ERR_INVALID_ARG), (dict(io_dtype=la.LA_FP8_E4M3), la.LA_ERR_INVALID_ARG),
    (dict(magnitude=float("nan")), la.LA_ERR_INVALID_ARG), (dict(turns_dev=None), la.LA_ERR_INVALID_ARG),
    (dict(n=-1), la.LA_ERR_INVALID_ARG), (dict(n=1 << 31), la.LA_ERR_INVALID_ARG),
], ids=str)
def test_plans_are_refused(change, want):
    assert _apply(**change) == want


@pytest.mark.parametrize("rows", [(None, P, 4, 0, 0), (P, None, 4, 0, 0), (P + 8, P, 4, 0, 0), (P, P + 2, 4, 0, 0),
                                  (P, P + 64, 0, 0, 0), (P, P + 64, -1, 0, 0), (P, P + 64, 4, 511, 0), (P, P + 64, 4, 0, 516),
                                  (P, P + 64, 4, 1 << 25, 0), (P, P, 4, 512, 520)], ids=str)
def test_rows_are_refused(rows):
    assert _apply(q=la.LaRopeRows(*rows)) == la.LA_ERR_INVALID_ARG
    assert _apply(k=la.LaRopeRows(*rows)) == la.LA_ERR_INVALID_ARG


def test_positions_are_refused():
    assert LIB.la_rope_apply(None, None, None, 1, None, 0, None) == la.LA_ERR_INVALID_ARG
    plan, q = la.LaRopePlan(128, 128, 0, la.LA_BF16, 1.0, P), la.LaRopeRows(P, P, 4, 0, 0)
    assert LIB.la_rope_apply(ctypes.byref(plan), ctypes.byref(q), None, 5, None, 0, None) == la.LA_ERR_INVALID_ARG
    for at in ((None, None, 2, P), (None, P, 2, None), (P, None, -1, None)):
        assert _apply(at=la.LaRopePositions(*at)) == la.LA_ERR_INVALID_ARG
    assert _apply(n=0, turns_dev=None) == la.LA_OK                # nothing to do
    assert _apply(at=la.LaRopePositions(None, None, 0, None)) == la.LA_OK
