"""Decode groups: empty ones and many of them, cache types behind max_group, and own keys around the
ends of a part (256 keys), against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

from test_gpu_attn import TYPES, Cache, _check, _host, _rand

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def _ref(q, cache, d):
    return [(i, oa.attend(_host(q[i:i + 1]), *cache.rows(i), n - 1, float(np.float32(d ** -0.5))), max(n, 1))
            for i, n in enumerate(cache.kv)]


@pytest.mark.parametrize("io,kind", [("bf16", "bf16"), ("f32", "f32")])
def test_groups_that_are_empty_at_first(io, kind):
    """Two empty groups when the plan is made; later the first three sequences share a prefix."""
    gen = torch.Generator().manual_seed(71)
    kv, d = [300, 290, 301, 40], 64
    cache = Cache(gen, kv, 2, d, kind, 16, shared=[(0, 3, 288)])
    q = _rand(gen, 4, 8, d).to(TYPES[io]).cuda()
    cu, pre, kv_dev = _i32([0, 0, 0]), _i32([288, 0]), _i32(kv)
    plan = api.AttnDecode(4, 8, 2, d, 301, TYPES[io], cu_group=cu, max_prefix_len=288)
    for groups in ([0, 0, 0], [0, 3, 3], [0, 3, 4], [4, 4, 4]):
        cu.copy_(_i32(groups))
        plan.workspace.fill_(0xFF)                   # a slot that nothing wrote is NaN
        o = plan.run(cache.layer(), q, kv_dev, pre)
        torch.cuda.synchronize()
        assert int(cache.err) == 0
        _check(o, _ref(q, cache, d), d, io == "bf16", f"groups {groups}, {kind}")
    # groups that are said to be empty share nothing, whatever cu_group holds
    cu.copy_(_i32([0, 3, 4]))
    none = la.make_prefix_groups(cu, pre, 0, 288)
    plan.workspace.fill_(0xFF)
    la.la_attn_decode(plan.shape, cache.layer(), q, kv_dev, 301, plan.o, none, plan.workspace)
    _check(plan.o, _ref(q, cache, d), d, io == "bf16", f"max_group 0, {kind}")


@pytest.mark.parametrize("io,kind,d", [("bf16", "bf16", 128), ("bf16", "fp8", 64), ("f32", "f32", 128)])
@pytest.mark.parametrize("prefix", [0, 40, 256])
def test_own_keys_around_the_end_of_a_part(io, kind, d, prefix):
    """Own keys of 255 to 257 and 511 to 513 tokens, from their 16-token line on: whole, and behind a prefix."""
    gen = torch.Generator().manual_seed(72)
    line = prefix // 16 * 16
    kv = [line + n for n in (255, 256, 257, 511, 512, 513, 769)]
    cache = Cache(gen, kv, 2, d, kind, 16, shared=[(0, len(kv), prefix)] if prefix else [])
    q = _rand(gen, len(kv), 6, d).to(TYPES[io]).cuda()
    cu = _i32([0, len(kv)]) if prefix else None
    plan = api.AttnDecode(len(kv), 6, 2, d, max(kv), TYPES[io], cu_group=cu, max_prefix_len=prefix)
    plan.workspace.fill_(0xFF)
    o = plan.run(cache.layer(), q, _i32(kv), _i32([prefix]) if prefix else None)
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    _check(o, _ref(q, cache, d), d, io == "bf16", f"own keys behind {prefix}, {kind}")


@pytest.mark.parametrize("io,kind", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
def test_more_groups_than_a_wave_reads_at_once(io, kind):
    """150 groups (64 are read at a time) of one to three sequences, with prefixes of many lengths."""
    gen = torch.Generator().manual_seed(73)
    sizes = [1 + i % 3 for i in range(150)]
    starts = np.concatenate([[0], np.cumsum(sizes)])
    prefix = [16 * (1 + 7 * i % 20) - (i % 5 == 4) * 3 for i in range(150)]
    kv = [p + 1 + (11 * j + i) % 40 for i, (n, p) in enumerate(zip(sizes, prefix)) for j in range(n)]
    shared = [(int(a), n, p) for a, n, p in zip(starts, sizes, prefix)]
    cache = Cache(gen, kv, 2, 64, kind, 16, shared=shared)
    q = _rand(gen, len(kv), 4, 64).to(TYPES[io]).cuda()
    plan = api.AttnDecode(len(kv), 4, 2, 64, max(kv), TYPES[io], cu_group=_i32(starts), max_prefix_len=max(prefix))
    plan.workspace.fill_(0xFF)
    o = plan.run(cache.layer(), q, _i32(kv), _i32(prefix))
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    _check(o, _ref(q, cache, 64), 64, io == "bf16", f"150 groups, {kind}")


@pytest.mark.parametrize("io,kind,d", [("bf16", "fp8", 128), ("f32", "f32", 64)])
@pytest.mark.parametrize("most", [1, 4, 8])
def test_sequences_behind_max_group(io, kind, d, most):
    """A group larger than its plan says: the sequences behind read their whole keys themselves."""
    gen = torch.Generator().manual_seed(74)
    kv = [300 + 7 * i for i in range(9)]
    cache = Cache(gen, kv, 2, d, kind, 16, shared=[(0, 9, 288)])
    q = _rand(gen, 9, 16, d).to(TYPES[io]).cuda()
    plan = api.AttnDecode(9, 16, 2, d, max(kv), TYPES[io], cu_group=_i32([0, 9]), max_prefix_len=288, max_group=most)
    plan.workspace.fill_(0xFF)
    o = plan.run(cache.layer(), q, _i32(kv), _i32([288]))
    torch.cuda.synchronize()
    _check(o, _ref(q, cache, d), d, io == "bf16", f"max_group {most}, {kind}")


@pytest.mark.parametrize("io,kind", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
def test_a_prefix_length_past_its_members(io, kind):
    """Slots of a batch that are out of use (no key, no block) beside a prefix length
    that is still there, and members that end before it: keys that no sequence sees
    are neither read nor counted as missing."""
    gen = torch.Generator().manual_seed(75)
    kv, d = [0, 0, 0, 300, 310, 100, 90, 257, 256], 64
    cache = Cache(gen, kv, 2, d, kind, 16, shared=[(3, 2, 288), (5, 2, 90)])
    q = _rand(gen, len(kv), 8, d).to(TYPES[io]).cuda()
    plan = api.AttnDecode(len(kv), 8, 2, d, 310, TYPES[io], cu_group=_i32([0, 3, 5, 7, 9]), max_prefix_len=288)
    plan.workspace.fill_(0xFF)
    cache.table[8] = cache.table[7]                  # the last group: one block is seen by its first member alone
    cache.table_dev.copy_(cache.table)
    o = plan.run(cache.layer(), q, _i32(kv), _i32([288, 288, 288, 257]))
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    assert not bool(o[:3].any())
    _check(o, _ref(q, cache, d), d, io == "bf16", f"prefix lengths past their members, {kind}")
