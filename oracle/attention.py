"""Attention and cache writes in fp64 NumPy, token by token from the definition.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Per token and query head h, with key head h // G and position x of the token:
s_j = scale <q, k_j> over the visible keys j <= x, j < kv_len; p = exp(s - max s);
o = sum p v / sum p.  No visible key: o = 0.
"""
from __future__ import annotations

import numpy as np

U16 = 2.0 ** -8        # rounding to bf16 (8 significant bits): half an ulp, relative
U32 = 2.0 ** -24


def attend(q, k, v, first, scale):
    """One sequence: q [n, Hq, d] at positions first, first + 1, ...; k, v
    [L, Hkv, d].  Returns (o, bound): bound[n, Hq, d] is how far a correct
    fp32 kernel may be off before its output is rounded, per unit of the
    weights' own rounding (see tolerance)."""
    n, Hq, d = q.shape
    L, Hkv, _ = k.shape
    o = np.zeros((n, Hq, d))
    mean = np.zeros((n, Hq, d))        # sum p |v| / sum p
    size = np.zeros((n, Hq, 1))        # most sum |q||k| scale of a visible key
    for t in range(n):
        seen = max(0, min(L, first + t + 1))
        if seen == 0:
            continue
        for h in range(Hq):
            kk, vv = k[:seen, h // (Hq // Hkv)], v[:seen, h // (Hq // Hkv)]
            s = scale * (kk @ q[t, h])
            if np.max(s) == -np.inf:
                continue
            p = np.exp(s - np.max(s))
            o[t, h] = (p @ vv) / p.sum()
            mean[t, h] = (p @ np.abs(vv)) / p.sum()
            size[t, h] = scale * np.max(np.abs(kk) @ np.abs(q[t, h]))
    return o, mean, size


def tolerance(o, mean, size, keys, d, bf16):
    """Absolute bound of each output.  Rounding the weights to bf16 moves the
    quotient by at most U16 of sum p |v| / sum p; an fp32 score of d terms is off
    by at most (d + 4) U32 of sum |q||k| scale, which moves a weight by that
    relative amount, in numerator and denominator; fp32 sums over the keys add
    2 keys U32 and the exponentials, rescalings and joins at most 32 U32; the
    output's rounding is half an ulp of its type (its error included: 1 %)."""
    up, uo = (U16, U16) if bf16 else (0.0, U32)
    e = mean * (up + 2 * (d + 4) * U32 * size + (2 * keys + 32) * U32)
    return e * 1.01 + uo * 1.01 * np.abs(o) + 1e-37


def table_rows(part, table, seq, n, bt, scale):
    """Keys or values [n, H, d] of a sequence from a layer's blocks [blocks, H,
    bt, d]; blocks that the table does not name hold zeros."""
    out = np.zeros((n, part.shape[1], part.shape[3]))
    for x in range(n):
        b = int(table[seq, x // bt])
        if 0 <= b < part.shape[0]:
            out[x] = part[b, :, x % bt] * scale
    return out
