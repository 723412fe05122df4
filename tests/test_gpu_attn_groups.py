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
