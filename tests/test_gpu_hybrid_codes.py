"""The example of examples/hybrid_request.py with rotary positions and a cache of 8-bit
codes: positions, writes, attention over the cache, forks and compaction as one run.

The oracle follows each sequence's blocks by themselves (their ids do not matter): what
each call writes is quantised as oracle.kv_codes does it, a fork begins with its parent's
codes and scales, and attention is fp64 over what they stand for (bound:
oracle.attention.tolerance).  Queries and keys are turned by la_rope_apply, which has
tests of its own, so that both sides quantise the same bf16 values."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import kv_codes as kc
from paper_2609_15030_amd import api

from parity import host
from test_gpu_hybrid_request import _example

pytestmark = pytest.mark.gpu


class Row:
    """One sequence's codes and scales, blocks in order."""

    def __init__(self, s, blocks):
        self.s, self.table = s, np.arange(blocks)[None, :]
        self.code = [np.zeros((blocks, s.kv_heads, s.block_tokens, s.head_dim)) for _ in (0, 1)]
        self.scale = [np.zeros((blocks, s.kv_heads)) for _ in (0, 1)]

    def fork(self):
        r = Row(self.s, self.table.shape[1])
        r.code, r.scale = [x.copy() for x in self.code], [x.copy() for x in self.scale]
        return r

    def write(self, k, v, end):
        for half, x in ((0, k), (1, v)):
            kc.write(self.code[half], self.scale[half], self.table, self.s.block_tokens, self.s.cache, x, [0, len(x)], [end])

    def rows(self, n):
        """Keys and values [n, heads, d]."""
        return [(c * s[:, :, None, None]).transpose(0, 2, 1, 3).reshape(-1, self.s.kv_heads, self.s.head_dim)[:n]
                for c, s in zip(self.code, self.scale)]


def _check(o, q, k, v, first, what):
    d = q.shape[2]
    ref, mean, size = oa.attend(q, k, v, first, float(np.float32(d ** -0.5)))
    off = np.abs(host(o) - ref) / oa.tolerance(ref, mean, size, k.shape[0], d, True)
    print(f"[hybrid codes] {what}: worst {off.max():.3f} of the bound", flush=True)
    assert off.max() <= 1.0, what


@pytest.mark.parametrize("sizes", [
    dict(prompt=520, shared=300, second=450, samples=3, steps=5, cache="int8", rotary=128),
    dict(prompt=300, shared=256, second=330, samples=2, steps=20, cache="e4m3", rotary=64, block_tokens=16),
    dict(prompt=270, shared=20, second=100, samples=1, steps=3, cache="int8", block_tokens=256, kv_heads=8),
], ids=lambda s: f"{s['cache']}-{s.get('rotary', 0)}-b{s.get('block_tokens', 64)}")
def test_requests_through_a_cache_of_codes(sizes):
    ex = _example()
    s = ex.Sizes(**sizes)
    r = ex.serve(s)
    hq, hk, bt = s.q_heads, s.kv_heads, s.block_tokens
    rope = api.Rope(s.head_dim, s.rotary) if s.rotary else None

    def split(t, first):
        t = t.clone()
        if rope:
            rope.apply(t[:, :hq], t[:, hq:hq + hk], positions=torch.arange(first, first + len(t), dtype=torch.int32, device="cuda"))
        x = host(t)
        return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]

    B = r["boundary"]
    assert B == s.shared // s.interval * s.interval and r["errors"] == 0
    blocks = -(-(max(s.prompt, s.second) + s.steps) // bt)
    q, k, v = split(r["first"].qkv, 0)
    _check(r["attn_first"][-50:], q[-50:], k, v, s.prompt - 50, "cold prompt, its last tokens")
    first = Row(s, blocks)
    first.write(k, v, s.prompt)
    q, k, v = split(r["second"].qkv[B:], B)
    second = first.fork()                                        # whole blocks up to B
    second.write(k, v, s.second)
    _check(r["attn_second"], q, *second.rows(s.second), B, "resumed prompt")
    for j in range(s.samples):
        row = second.fork()
        for i, t in enumerate(r["steps"]):
            n = s.second + i + 1
            q, k, v = split(t.qkv[j:j + 1], n - 1)
            row.write(k, v, n)
            _check(r["attn_steps"][i, j][None], q, *row.rows(n), n - 1, f"sample {j}, step {i}")
    whole, last = s.second // bt, -(-(s.second + s.steps) // bt)
    assert r["blocks"] - r["free"] == -(-s.second // bt) + s.samples * (last - whole)
