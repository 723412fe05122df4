"""Attention over int8 codes whose key scale times the softmax scale lies below fp32's
normal numbers: scores are still what they should be, and masked keys weigh nothing.

The factor of a score, of at least 2^-149, is off by at most that, and a sum of products
that fp32 holds is below 2^128: a score in base 2 is off by 2^-21 from it, a weight so by
2^-21, in numerator and denominator, besides what the oracle's bound has."""
import numpy as np
import pytest
import torch

from codes import CodeCache, tables
from oracle import attention as oa
from paper_2609_15030_amd import api

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -100


def _host(t):
    return t.detach().double().cpu().numpy()


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _check(o, q, cache, new, kv, scale, what):
    got, at, d = _host(o), 0, q.shape[2]
    assert np.all(np.isfinite(got)), what
    for i, (n, L) in enumerate(zip(new, kv)):
        ref, mean, size = oa.attend(_host(q[at:at + n]), cache.rows(i, L, 0), cache.rows(i, L, 1), L - n, scale)
        tol = oa.tolerance(ref, mean, size, L, d, True) + 2 * 2.0 ** -21 * mean
        worst = float(np.max(np.abs(got[at:at + n] - ref) / tol, initial=0.0))
        print(f"[small scales] {what} {i}: worst {worst:.3f} of the bound", flush=True)
        assert worst <= 1.0, (what, i, worst)
        at += n


@pytest.mark.parametrize("power", [-26, -30, -47, -60, -125])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_below_the_normal_numbers(d, power):
    """Queries of such a size that a factor of 2^-126 would give one key about twice the others' weight."""
    scale = 2.0 ** power
    gen = torch.Generator().manual_seed(74)
    kv, new, hq, bt = [40, 9, 700, 41], [40, 3, 30, 1], 2, 16
    table, blocks = tables(gen, kv, bt)
    c = CodeCache(gen, "int8", 1, d, bt, table, blocks)
    code, s = c.numbers(0)
    c.put(0, code, np.full_like(s, LEAST))
    c.dev.copy_(c.bytes)
    size = 2.0 ** 121 / d                                                   # sums of products: below 2^128
    along = np.stack([np.sign(code[table[i, 0], 0, 1]) for i in range(4)])    # each sequence's second key
    of = lambda i: torch.from_numpy(np.stack([along[i], -along[i]]) * size).to(torch.bfloat16)
    q = torch.cat([of(i)[None].expand(n, hq, d) for i, n in enumerate(new)]).cuda()
    o = api.AttnPrefill(hq, 1, d, new, kv, scale=scale).run_paged(c.layer(), q)
    torch.cuda.synchronize()
    _check(o, q, c, new, kv, scale, f"prompts {d} 2^{power}")
    rows = torch.stack([of(i) for i in range(4)]).cuda()
    o = api.AttnDecode(4, hq, 1, d, max(kv), scale=scale).run(c.layer(), rows, _i32(kv))
    torch.cuda.synchronize()
    _check(o, rows, c, [1] * 4, kv, scale, f"single tokens {d} 2^{power}")
    c.table[1:, 0] = c.table[0, 0]                                          # a prefix of one block
    c.table[1, 1] = c.table[2, 1]
    c.table_dev = torch.from_numpy(c.table).cuda()
    rows, kv = of(0)[None].repeat(4, 1, 1).cuda(), [40, 25, 700, 41]
    plan = api.AttnDecode(4, hq, 1, d, max(kv), scale=scale, cu_group=_i32([0, 4]), max_prefix_len=16)
    o = plan.run(c.layer(), rows, _i32(kv), _i32([16]))
    torch.cuda.synchronize()
    _check(o, rows, c, [1] * 4, kv, scale, f"shared prefix {d} 2^{power}")
    assert int(c.err) == 0
