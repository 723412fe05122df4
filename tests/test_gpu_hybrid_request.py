"""The example of examples/hybrid_request.py as a test: a cold prompt, a prompt
resumed from its blocks and states, and samples that decode together while the
first prompt is retired.

Attention is compared with fp64 attention over each sequence's own tokens, laid
out without any cache (bound: oracle.attention.tolerance); the resumed recurrent
outputs with a cold run's suffix, bit for bit; the decoded ones with the fp64
recurrence.  Block counts are worked out from the lengths.
"""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from oracle import attention as oa
from paper_2609_15030_amd import api

from parity import TOL, host, slice_err

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_request.py")
    spec = importlib.util.spec_from_file_location("hybrid_request", path)
    module = sys.modules[spec.name] = importlib.util.module_from_spec(spec)      # its dataclasses look themselves up
    spec.loader.exec_module(module)
    return module


def _check(o, q, k, v, first, what):
    d = q.shape[2]
    ref, mean, size = oa.attend(q, k, v, first, d ** -0.5)
    off = np.abs(host(o) - ref) / oa.tolerance(ref, mean, size, k.shape[0], d, True)
    print(f"[hybrid request] {what}: worst {off.max():.3f} of the bound", flush=True)
    assert off.max() <= 1.0, what


@pytest.mark.parametrize("sizes", [
    dict(prompt=700, shared=600, second=650, samples=3, steps=6),
    dict(prompt=520, shared=256, second=513, samples=1, steps=2, block_tokens=16),
    dict(prompt=300, shared=200, second=448, samples=5, steps=4, kv_heads=8),       # no common checkpoint: B = 0
])
def test_requests_through_one_cache(sizes):
    ex = _example()
    s = ex.Sizes(**sizes)
    r = ex.serve(s)
    hq, hk = s.q_heads, s.kv_heads

    def split(t):
        x = host(t)
        return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]

    B = r["boundary"]
    assert B == (s.shared // s.interval) * s.interval and r["errors"] == 0
    _check(r["attn_first"], *split(r["first"].qkv), 0, "cold prompt")
    q, k, v = split(r["second"].qkv)
    _check(r["attn_second"], q[B:], k, v, B, "resumed prompt")
    cold = api.prefill(api.to_device(r["second"].rec), s.interval, emit_ckpt=False)
    assert torch.equal(r["rec_second"], cold.o[B:])

    state = oracle.gdr_prefill_seq(*[getattr(r["second"].rec, f) for f in ("q", "k", "v", "g", "beta")])[1]
    for j in range(s.samples):
        own = [split(t.qkv[j:j + 1]) for t in r["steps"]]
        kj = np.concatenate([k] + [x[1] for x in own])
        vj = np.concatenate([v] + [x[2] for x in own])
        _check(r["attn_steps"][:, j], np.concatenate([x[0] for x in own]), kj, vj, s.second, f"sample {j}")
        rec = [np.concatenate([getattr(t.rec, f)[j:j + 1] for t in r["steps"]]) for f in ("q", "k", "v", "g", "beta")]
        ref = oracle.gdr_prefill_seq(*rec, state_in=state)[0]
        got = host(r["rec_steps"][:, j])
        assert max(slice_err(got[:, h], ref[:, h]) for h in range(s.heads)) <= TOL[api.la.LA_BF16]

    # the retired prompt leaves what the second one shares; the samples share its whole blocks
    bt = s.block_tokens
    whole, last = s.second // bt, -(-(s.second + s.steps) // bt)
    assert r["blocks"] - r["free"] == -(-s.second // bt) + s.samples * (last - whole)
