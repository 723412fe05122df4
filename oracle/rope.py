"""Rotary positions in fp64 (angles in extended precision), pair by pair as complex numbers.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(rotary, base, kind=None, factor=1.0, original=0.0, low=0.0, high=0.0):
    """Radians a token of each pair, one at a time."""
    out = []
    for i in range(rotary // 2):
        b = base * factor ** (rotary / (rotary - 2)) if kind == "base" and rotary > 2 else base
        f = b ** (-2 * i / rotary)
        if kind == "linear":
            f /= factor
        if kind == "parts":
            n = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (n - low) / (high - low)))
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out)


def turn(x, pos, freq, layout, magnitude=1.0, transpose=False):
    """x [T, heads, d] at positions pos [T]."""
    y = np.array(x, np.float64)
    r = 2 * len(freq)
    turn_of = np.longdouble("6.283185307179586476925286766559")
    for i, f in enumerate(freq):
        a, b = (i, i + r // 2) if layout == "halves" else (2 * i, 2 * i + 1)
        angle = np.fmod(np.asarray(pos, np.longdouble) * np.longdouble(f), turn_of).astype(np.float64)     # off by 1e-9 at 2^31
        w = magnitude * np.exp((-1j if transpose else 1j) * angle)
        z = (y[:, :, a] + 1j * y[:, :, b]) * w[:, None]
        y[:, :, a], y[:, :, b] = z.real, z.imag
    return y
