"""Caches of 8-bit codes and rotary positions at the ends of what the entry points
accept: blocks, lengths and launches whose offsets pass 32 bits, scores past fp32's range."""
import numpy as np
import pytest
import torch

from codes import TYPES, CodeCache
from oracle import attention as oa
from oracle import kv_codes as kc
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu
KINDS = ["e4m3", "int8"]


def _host(t):
    return t.detach().double().cpu().numpy()


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _check(o, q, k, v, first, what):
    d = q.shape[2]
    ref, mean, size = oa.attend(_host(q), k, v, first, float(np.float32(d ** -0.5)))
    off = np.abs(_host(o) - ref) / oa.tolerance(ref, mean, size, k.shape[0], d, True)
    print(f"[codes limits] {what}: worst {off.max():.3f} of the bound", flush=True)
    assert off.max() <= 1.0, what


@pytest.mark.parametrize("kind", KINDS)
def test_a_layer_whose_keys_take_over_2_gb_of_a_block(kind):
    """The last heads of a block begin past 2^31 bytes behind its keys."""
    d, bt, heads, n = 128, 256, 65600, 3
    part = heads * bt * d
    assert part > 1 << 31
    cache = torch.empty((1, 2 * part + 8 * heads), dtype=torch.uint8, device="cuda")
    layer = la.make_kv_layer(cache, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), bt, heads, d, TYPES[kind],
                             k_scales=2 * part)
    gen = torch.Generator(device="cuda").manual_seed(61)
    q, k, v = (torch.randn((n, heads, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    cu, kv = _i32([0, n]), _i32([n])
    la.la_kv_write(layer, k, v, cu, kv)
    yk, yv = torch.empty_like(k, dtype=torch.float32), torch.empty_like(v, dtype=torch.float32)
    la.la_kv_read(layer, yk, yv, cu, kv)
    got = api.AttnPrefill(heads, heads, d, [n], [n]).run_paged(layer, q)
    one = api.AttnDecode(1, heads, heads, d, n).run(layer, q[n - 1:], kv)
    torch.cuda.synchronize()
    some = [0, heads // 2, heads - 17, heads - 1]
    kept = []
    for x, y in ((k, yk), (v, yv)):
        x, want = _host(x[:, some]), []
        for i in range(len(some)):
            s = kc.scale_of(np.abs(x[:, i]).max(), kind)
            want.append(kc.codes(x[:, i] / s, kind) * s)
        kept.append(np.stack(want, 1))
        assert np.array_equal(_host(y[:, some]), kept[-1])
    _check(got[:, some], q[:, some], *kept, 0, f"{heads} heads, prompt")
    _check(one[:, some], q[n - 1:][:, some], *kept, n - 1, f"{heads} heads, single token")


@pytest.mark.parametrize("kind", KINDS)
def test_the_longest_sequence(kind):
    """2^31 - 256 keys, all but the last block's in one block of zero keys and equal values: the first
    query head sees the last block alone (its keys score 64 more), the second the others, whose sums are exact."""
    d, bt, last = 64, 256, 0x7FFFFF00
    gen = torch.Generator().manual_seed(62)
    c = CodeCache(gen, kind, 1, d, bt, np.array([[0, 1]]), 2, layers=1)
    k = 0.02 * torch.randn((bt, 1, d), generator=gen)
    k[..., 0] = 16.0
    v = torch.randn((bt, 1, d), generator=gen)
    whole = torch.arange(d) % 4 + 1
    for half, x in ((0, torch.zeros(bt, 1, d)), (1, whole.expand(bt, 1, d))):
        code, scale = c.numbers(half)
        code[0] = x.double().permute(1, 0, 2).numpy()
        scale[0] = 1.0
        c.put(half, code, scale)
    c.table = np.array([[1]])
    c.write(k.to(torch.bfloat16), v.to(torch.bfloat16), [0, bt], [bt])
    c.dev.copy_(c.bytes)
    table = torch.zeros((1, last // bt), dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    layer = la.make_kv_layer(c.dev, table, bt, 1, d, TYPES[kind], c.off[0], c.off[1], err_count=c.err,
                             k_scales=c.scales_at[0], v_scales=c.scales_at[1])
    q = torch.zeros((1, 2, d), device="cuda")
    q[0, :, 0] = torch.tensor([32.0, -32.0], device="cuda")               # scores: about +-32 x 16 / 8
    q = q.to(torch.bfloat16)
    for what, o in (("prompt", api.AttnPrefill(2, 1, d, [1], [last]).run_paged(layer, q)),
                    ("single token", api.AttnDecode(1, 2, 1, d, last).run(layer, q, _i32([last])))):
        torch.cuda.synchronize()
        assert int(c.err) == 0
        _check(o[:, :1], q[:, :1], c.rows(0, bt, 0), c.rows(0, bt, 1), bt - 1, f"longest sequence, {what}")
        off = (o[0, 1].double().cpu() - whole).abs() / whole
        assert float(off.max()) <= 2 ** -8, (what, float(off.max()))


@pytest.mark.parametrize("kind", KINDS)
def test_writes_of_more_workgroups_than_a_launch_has(kind):
    """2^32 threads are 2^24 workgroups; two for each of 2^23 sequences, all empty but the last thousand."""
    n, some, d, bt = (1 << 23) + 1000, 1000, 64, 16
    gen = torch.Generator().manual_seed(63)
    k, v = (torch.randn((some, 1, d), generator=gen).to(torch.bfloat16).cuda() for _ in (0, 1))
    cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    cu[n - some:] = torch.arange(some + 1, dtype=torch.int32, device="cuda")
    table = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
    table[n - some:, 0] = torch.arange(some, dtype=torch.int32, device="cuda")
    kv = torch.zeros(n, dtype=torch.int32, device="cuda")
    kv[n - some:] = 1
    c = CodeCache(gen, kind, 1, d, bt, np.arange(some)[:, None], some, layers=1)
    layer = la.make_kv_layer(c.dev, table, bt, 1, d, TYPES[kind], c.off[0], c.off[1], err_count=c.err,
                             k_scales=c.scales_at[0], v_scales=c.scales_at[1])
    la.la_kv_write(layer, k, v, cu, kv)
    torch.cuda.synchronize()
    c.write(k, v, range(some + 1), [1] * some)
    c.same(kind)
    assert int(c.err) == 0


def test_rotations_of_more_tokens_than_a_launch_takes():
    """Tokens behind the first launch's 33,554,400 have the bits that a call of their own gives."""
    n, d = 33554400 + 1000, 8
    x = torch.randn((n, 1, d), device="cuda", dtype=torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rope, y = api.Rope(d), torch.empty_like(x)
    rope.apply(x, None, y, positions=pos)
    for a in (0, 33554400 - 500, n - 700):
        z = torch.empty_like(x[a:a + 700])
        rope.apply(x[a:a + 700], None, z, positions=pos[a:a + 700].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(y[a:a + 700], z), a


@pytest.mark.parametrize("kind", KINDS)
def test_scores_past_the_range_of_fp32(kind):
    """Tokens that see one have NaN, those before it are as they were, and one of minus infinity weighs
    nothing: prompts, single tokens and a shared prefix."""
    d, n, bt, key = 64, 150, 16, 100
    gen = torch.Generator().manual_seed(64)
    blocks = -(-n // bt)
    c = CodeCache(gen, kind, 1, d, bt, np.arange(blocks)[None].repeat(3, 0), blocks, layers=1)
    q = 2.0 ** -10 * torch.randn((n, 2, d), generator=gen)
    k, v = torch.randn((n, 1, d), generator=gen), torch.randn((n, 1, d), generator=gen)
    q[..., 0], k[..., 0] = 0, 0
    q, k, v = (x.to(torch.bfloat16).cuda() for x in (q, k, v))
    one, big = _i32([0, n]), 2.0 ** 10
    la.la_kv_write(c.layer(), k, v, one, _i32([n]))
    plan = api.AttnPrefill(2, 1, d, [n], [n], scale=big)
    clean = plan.run_paged(c.layer(), q).clone()
    # one key of its own scale: 16 tokens of its block hold nothing else of that size
    code, scale = c.numbers(0, c.dev.cpu())
    b = key // bt
    c.bytes.copy_(c.dev.cpu())
    code[b], scale[b] = 0.0, 2.0 ** 55
    code[b, 0, key % bt, 0] = 32.0                                         # 2^60
    c.put(0, code, scale)
    c.dev.copy_(c.bytes)
    q2 = q.clone()
    q2[:, 0, 0], q2[:, 1, 0] = 2.0 ** 60, -2.0 ** 60
    o = plan.run_paged(c.layer(), q2)
    torch.cuda.synchronize()
    assert torch.equal(o[:b * bt], clean[:b * bt])
    assert torch.isnan(o[key:, 0]).all() and torch.isfinite(o[key:, 1]).all()
    kk, vv = c.rows(0, n, 0), c.rows(0, n, 1)
    rest = [j for j in range(n) if j != key]
    ref, mean, size = oa.attend(_host(q[n - 1:, 1:]), kk[rest], vv[rest], n - 2, big)
    tol = oa.tolerance(ref, mean, size, n, d, True)
    assert np.all(np.abs(_host(o[n - 1:, 1:]) - ref) <= tol)
    kv, rows = torch.full((3,), n, dtype=torch.int32, device="cuda"), q2[n - 3:].contiguous()
    for groups in (None, _i32([0, 3])):
        dec = api.AttnDecode(3, 2, 1, d, n, scale=big, cu_group=groups, max_prefix_len=0 if groups is None else 144)
        t = dec.run(c.layer(), rows, kv, None if groups is None else _i32([144]))
        torch.cuda.synchronize()
        assert torch.isnan(t[:, 0]).all() and torch.isfinite(t[:, 1]).all()
        assert np.all(np.abs(_host(t[2:, 1:]) - ref) <= tol)
