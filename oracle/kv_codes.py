"""A cache of 8-bit codes with a scale for each block and head, in fp64 NumPy and
exact fractions, token by token from the definition.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Codes are kept as the numbers they are (float64): e4m3 values, or integers.
NaN is NaN; int8 has none.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

LEAST = Fraction(1, 2 ** 100)
LARGEST = 2.0 ** 127                  # what lies beyond is written as this

# the finite e4m3 numbers from 0 up: 3 bits of mantissa, exponents -6 to 8, subnormals below, 480 left to NaN
E4M3 = np.array([m / 8 * 2.0 ** -6 for m in range(8)] +
                [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])


def e4m3(x):
    """Nearest e4m3 numbers, ties to the even one (of |x| <= 448)."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isnan(x), 0.0, np.abs(x))
    hi = np.searchsorted(E4M3, a).clip(max=len(E4M3) - 1)      # first one not below
    lo = np.maximum(hi - (E4M3[hi] > a), 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    pick = np.where(up < down, hi, np.where(up > down, lo, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(x), np.nan, np.copysign(E4M3[pick], x))


def bf16(x):
    """Nearest bf16 numbers of fp64 values, ties to the even one."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x)
    unit = np.ldexp(1.0, np.maximum(np.frexp(np.where(finite, x, 0.0))[1] - 8, -133))       # of the last of 8 significant bits
    y = np.rint(np.where(finite, x, 0.0) / unit) * unit
    y = np.where(np.abs(y) >= 2.0 ** 128, np.copysign(np.inf, y), y)
    return np.where(finite, y, x)


def codes(x, kind):
    return e4m3(x) if kind == "e4m3" else np.rint(np.where(np.isnan(x), 0.0, x))


def scale_of(most: float, kind: str) -> float:
    """The scale that values up to `most` ask for."""
    a = Fraction(float(most))
    if kind == "e4m3":
        s = LEAST
        while a > 448 * s:
            s *= 2
        return float(s)
    s = a / 127
    if s <= LEAST:
        return float(LEAST)
    step = LEAST                       # a unit of the last of 8 significant bits
    while s > 256 * step:
        step *= 2
    while s <= 128 * step:
        step /= 2
    return float(-(-s // step) * step)


def held(s: float, kind: str) -> float:
    """A block's scale as a later write sees it: one that no write can have left is the least."""
    s = float(s)
    if not (float(LEAST) <= s <= scale_of(LARGEST, kind)):
        return float(LEAST)
    m = Fraction(s)
    while m >= (2 if kind == "e4m3" else 256):
        m /= 2
    while m < (1 if kind == "e4m3" else 128):
        m *= 2
    return s if m.denominator == 1 else float(LEAST)


def write(code, scale, table, bt, kind, x, cu, kv, first=0):
    """Writes rows x [T, H, d] (keys or values) of the sequences into code
    [blocks, H, bt, d] and scale [blocks, H], in place; positions that have no
    block are skipped."""
    x = np.where(np.isnan(x), np.nan, np.clip(x, -LARGEST, LARGEST))
    blocks, H = scale.shape
    for i in range(len(kv)):
        n = int(cu[i + 1]) - int(cu[i])
        start = int(kv[i]) - n
        by_block = {}
        for t in range(n):
            p = start + t
            j = p // bt
            b = int(table[i][j]) if 0 <= j < table.shape[1] else -1
            if p >= 0 and 0 <= b < blocks:
                by_block.setdefault(b, []).append((p % bt, int(cu[i]) + t))
        for b, rows in by_block.items():
            a0 = rows[0][0]
            for h in range(H):
                y = np.stack([x[t, h] for _, t in rows])
                seen = np.abs(y[~np.isnan(y)])
                s = scale_of(seen.max() if seen.size else 0.0, kind)
                if a0 > 0:
                    old = held(scale[b, h], kind)
                    if s > old:
                        code[b, h, :a0] = codes(code[b, h, :a0] * (old / s) if kind == "e4m3" else code[b, h, :a0] * old / s, kind)
                    s = max(s, old)
                scale[b, h] = s
                for slot, t in rows:
                    code[b, h, slot] = codes(x[t, h] / s, kind)
