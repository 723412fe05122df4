"""Prompt calls that fill the chip: sequences whole rather than in parts, the longest
first, over key loops that pass 1,024 tokens of a block table twice.  Every row
against attention in fp64 (two-dimensional products, one head at a time), with the
bound of oracle/attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

from test_gpu_attn import TYPES, Cache, _host, _rand

pytestmark = pytest.mark.gpu

# Rows of a workgroup, and the workgroups above which a call takes long sequences first.
TILE = {"bf16": 128, "f32": 64}
FULL = {"bf16": 512, "f32": 2048}


def _attend64(q, k, v, first, scale):
    """(o, mean, size) of oracle.attention.attend for one sequence of device tensors."""
    q, k, v = (x.to(torch.float64) for x in (q, k, v))
    n, hq, d = q.shape
    L, hk = k.shape[:2]
    o, mean, size = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((n, hq, 1), dtype=torch.float64, device=q.device)
    seen = torch.arange(L, device=q.device)[None, :] <= first + torch.arange(n, device=q.device)[:, None]
    some = seen.any(1)
    for h in range(hq):
        kk, vv = k[:, h // (hq // hk)], v[:, h // (hq // hk)]
        s = (scale * (q[:, h] @ kk.T)).masked_fill(~seen, -torch.inf)
        p = torch.exp(s - s.amax(1, keepdim=True).clamp(min=-1e300))
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        o[:, h], mean[:, h] = p @ vv, p @ vv.abs()
        size[:, h, 0] = (scale * (q[:, h].abs() @ kk.abs().T)).masked_fill(~seen, 0.0).amax(1)
    assert bool((o[~some] == 0).all())
    return tuple(x.cpu().numpy() for x in (o, mean, size))


def _check_every_row(o, new, keys, d, bf16, reference):
    """reference(i, at): (q, k, v) of sequence i, whose rows begin at `at`."""
    at, worst = 0, 0.0
    for i, (n, L) in enumerate(zip(new, keys)):
        if n:
            ref, mean, size = _attend64(*reference(i, at), L - n, float(np.float32(d ** -0.5)))
            off = np.abs(_host(o[at:at + n]) - ref) / oa.tolerance(ref, mean, size, max(L, 1), d, bf16)
            assert np.all(np.isfinite(off)), i
            worst = max(worst, float(off.max()))
        at += n
    print(f"[attn large] {len(new)} sequences, {at} rows: worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


def _fills_the_chip(new, group, kv_heads, io):
    tiles = sum(-(-n * group // TILE[io]) for n in new)
    return tiles * kv_heads > FULL[io] and 1 < len(new) <= 64


MANY = [2200] + [37 * i % 90 for i in range(1, 64)]

CALLS = [
    # new tokens, keys of the cache before them, q heads, kv heads, d, io, cache, block tokens
    ([2300, 0, 1, 700, 2600, 130, 64, 65, 1290, 900, 333, 40], [9, 7, 30, 2500, 0, 1000, 1, 63, 64, 129, 1700, 2048], 8, 4, 64,
     "bf16", "bf16", 16),
    (MANY, [211 * i % 1500 for i in range(64)], 16, 4, 128, "bf16", "fp8", 32),
    ([2200, 1, 2050], [100, 2300, 0], 16, 4, 128, "bf16", "bf16", 256),
    ([2300, 0, 1, 1500, 2100, 900, 700, 650, 400], [9, 7, 2500, 1000, 0, 129, 1, 2000, 64], 16, 4, 64, "f32", "f32", 16),
    ([4000, 3999, 2100, 6400, 1], [50, 0, 1024, 1, 900], 8, 8, 128, "f32", "f32", 64),
]


def _name(c):
    return f"{len(c[0])}x{max(c[0])}-{c[2]}/{c[3]}x{c[4]}-{c[6]}-b{c[7]}"


@pytest.mark.parametrize("case", CALLS, ids=_name)
def test_prompts_over_a_cache(case):
    new, before, hq, hk, d, io, kind, bt = case
    kv = [n + x for n, x in zip(new, before)]
    kv[0] -= 40 + before[0]                                    # more tokens than keys: the first see none
    assert _fills_the_chip(new, hq // hk, hk, io) and kv[0] > 2100      # three steps of 1,024 tokens of the table
    gen = torch.Generator().manual_seed(82)
    q, cache = _rand(gen, sum(new), hq, d).to(TYPES[io]).cuda(), Cache(gen, kv, hk, d, kind, bt)
    plan = api.AttnPrefill(hq, hk, d, new, kv, TYPES[io])
    assert plan.workspace.numel() == 16                        # whole rows: nothing to join
    plan.o.fill_(float("nan"))
    o = plan.run_paged(cache.layer(), q).clone()
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    assert torch.equal(plan.run_paged(cache.layer(), q), o)
    def reference(i, at):
        k, v = (torch.from_numpy(x).cuda() for x in cache.rows(i))
        return q[at:at + new[i]], k, v

    _check_every_row(o, new, kv, d, io == "bf16", reference)


@pytest.mark.parametrize("case", [c for c in CALLS if c[6] != "fp8"], ids=_name)
def test_packed_prompts(case):
    new, _, hq, hk, d, io, _, _ = case
    assert _fills_the_chip(new, hq // hk, hk, io) and max(new) > 2100
    gen = torch.Generator().manual_seed(84)
    x = _rand(gen, sum(new), hq + 2 * hk, d).to(TYPES[io]).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    plan = api.AttnPrefill(hq, hk, d, new, dtype=TYPES[io])
    assert plan.workspace.numel() == 16
    plan.o.fill_(float("nan"))
    o = plan.run(q, k, v)
    torch.cuda.synchronize()
    _check_every_row(o, new, new, d, io == "bf16", lambda i, at: tuple(y[at:at + new[i]] for y in (q, k, v)))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_missing_blocks_behind_the_first_1024_tokens(io):
    """Entries that name no block, in the second and third step of the table, read as zero and count."""
    new, kv, hq, hk, d, bt = [2400, 2500, 2000, 2600], [2450, 2500, 2300, 2600], 16, 4, 64, 16
    assert _fills_the_chip(new, hq // hk, hk, io)
    gen = torch.Generator().manual_seed(85)
    q, cache = _rand(gen, sum(new), hq, d).to(TYPES[io]).cuda(), Cache(gen, kv, hk, d, io, bt)
    for i, at, entry in ((0, 70, -1), (1, 130, cache.host.shape[0]), (2, 64, -3), (3, 127, -1)):
        cache.table[i, at] = entry
    cache.table_dev.copy_(cache.table)
    o = api.AttnPrefill(hq, hk, d, new, kv, TYPES[io]).run_paged(cache.layer(), q)
    torch.cuda.synchronize()
    assert int(cache.err) >= 4
    def reference(i, at):
        k, v = (torch.from_numpy(x).cuda() for x in cache.rows(i))
        return q[at:at + new[i]], k, v

    _check_every_row(o, new, kv, d, io == "bf16", reference)
