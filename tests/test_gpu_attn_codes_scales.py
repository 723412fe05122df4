"""Attention over codes whose blocks' scales lie at the ends of what a write can leave: keys of
tiny scale under large queries, keys of large scale under small ones, values of either, mixed in one sequence."""
import numpy as np
import pytest
import torch

from codes import CodeCache, tables
from oracle import attention as oa
from paper_2609_15030_amd import api

pytestmark = pytest.mark.gpu


def _host(t):
    return t.detach().double().cpu().numpy()


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _check(o, q, cache, new, kv, what):
    got, at, d = _host(o), 0, q.shape[2]
    assert np.all(np.isfinite(got)), what
    for i, (n, L) in enumerate(zip(new, kv)):
        ref, mean, size = oa.attend(_host(q[at:at + n]), cache.rows(i, L, 0), cache.rows(i, L, 1), L - n, float(np.float32(d ** -0.5)))
        worst = float(np.max(np.abs(got[at:at + n] - ref) / oa.tolerance(ref, mean, size, L, d, True), initial=0.0))
        print(f"[scales] {what} {i}: worst {worst:.3f} of the bound", flush=True)
        assert worst <= 1.0, (what, i, worst)
        at += n


# powers of two of the scales of keys and of values in even and in odd blocks
ENDS = [((-100, -100), (-6, -6)), ((100, 100), (-6, -6)), ((-6, -6), (-100, -100)), ((-6, -6), (105, 105)), ((-6, -6), (-100, -90)),
        ((-6, -6), (-20, 100)), ((-100, -94), (-3, -6))]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("ends", ENDS, ids=str)
def test_scales_at_the_ends(ends, kind):
    gen = torch.Generator().manual_seed(75)
    kv, new, hq, d, bt = [40, 9, 700], [40, 3, 30], 2, 128, 16
    table, blocks = tables(gen, kv, bt)
    c = CodeCache(gen, kind, 1, d, bt, table, blocks)
    odd = np.zeros((blocks, 1), bool)
    for row in table:
        odd[[b for b in row[1::2] if b >= 0]] = True
    size = np.abs(c.numbers(0)[0]).max() / 4                                # codes are of this size
    for half in (0, 1):
        code, s = c.numbers(half)
        c.put(half, code, np.where(odd, 2.0 ** ends[half][1], 2.0 ** ends[half][0]))
    c.dev.copy_(c.bytes)
    q = torch.randn((sum(new), hq, d), generator=gen, dtype=torch.float64) / size * 2.0 ** -max(ends[0])      # scores of a few units
    q = q.to(torch.bfloat16).cuda()
    o = api.AttnPrefill(hq, 1, d, new, kv).run_paged(c.layer(), q)
    torch.cuda.synchronize()
    _check(o, q, c, new, kv, f"prompts {ends} {kind}")
    rows = torch.stack([q[39], q[42], q[72]])
    o = api.AttnDecode(3, hq, 1, d, max(kv)).run(c.layer(), rows, _i32(kv))
    torch.cuda.synchronize()
    _check(o, rows, c, [1] * 3, kv, f"single tokens {ends} {kind}")
    c.table[1:, 0] = c.table[0, 0]                                          # a prefix of one block
    c.table[1, 1] = c.table[2, 1]
    c.table_dev = torch.from_numpy(c.table).cuda()
    kv = [40, 25, 700]
    plan = api.AttnDecode(3, hq, 1, d, max(kv), cu_group=_i32([0, 3]), max_prefix_len=16)
    o = plan.run(c.layer(), rows, _i32(kv), _i32([16]))
    torch.cuda.synchronize()
    _check(o, rows, c, [1] * 3, kv, f"shared prefix {ends} {kind}")
    assert int(c.err) == 0


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_groups_of_one_sequence_and_of_none(kind):
    """They share nothing, whatever prefix stands for them; their neighbours do."""
    gen = torch.Generator().manual_seed(76)
    kv, hq, d, bt = [300, 290, 333, 40, 17, 270, 280], 4, 64, 16
    table, blocks = tables(gen, kv, bt)
    table[1:3, :16] = table[1, :16]
    table[5:7, :16] = table[5, :16]
    c = CodeCache(gen, kind, 2, d, bt, table, blocks)
    q = torch.randn((7, hq, d), generator=gen).to(torch.bfloat16).cuda()
    cu = _i32([0, 1, 3, 3, 4, 5, 7])
    o = api.AttnDecode(7, hq, 2, d, max(kv), cu_group=cu, max_prefix_len=256).run(c.layer(), q, _i32(kv), _i32([256, 256, 256, 40, 16, 256]))
    torch.cuda.synchronize()
    _check(o, q, c, [1] * 7, kv, f"groups {kind}")
    assert int(c.err) == 0
