"""Quantising writes into caches with a scale for each block and head, and reads of
every kind of cache, against the fp64 oracle (oracle/kv_codes.py).

Codes and scales have to be the oracle's exactly: a scale has 8 significant bits,
a bf16 value 8, so that no quotient but a tie is within fp32's error of one.
Reads round a product that is exact in fp32 once: compared with its rounding."""
import numpy as np
import pytest
import torch

from codes import TYPES, CodeCache, tables
from oracle import kv_codes as kc
from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu
KINDS = ["e4m3", "int8"]


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _offsets(lens, first=0):
    return [first + sum(lens[:i]) for i in range(len(lens) + 1)]


def _rows(gen, T, H, d, stride_heads=0, spread=4.0):
    """Keys and values [T, H, d] in bf16, of magnitudes spread over tokens; slices of wider rows where stride_heads."""
    x = torch.randn((T, 2 * H + stride_heads, d), generator=gen, dtype=torch.float64)
    x *= 2.0 ** (spread * torch.rand((T, 1, 1), generator=gen, dtype=torch.float64))
    x = x.to(torch.bfloat16).cuda()
    k, v = x[:, :H], x[:, H:2 * H]
    return (k, v) if stride_heads else (k.contiguous(), v.contiguous())


WRITES = [
    # new tokens, kv after them, heads, d, block tokens
    ([1], [1], 1, 64, 16),
    ([1, 1, 1, 1], [16, 17, 5, 300], 3, 128, 16),
    ([5, 0, 40, 16], [21, 9, 57, 16], 2, 128, 16),
    ([31, 33], [31, 65], 5, 64, 32),
    ([100, 1, 7], [131, 64, 63], 2, 128, 32),
    ([200], [260], 2, 128, 64),
    ([1, 130, 3], [64, 130, 190], 1, 64, 64),
    ([300, 2], [301, 130], 3, 128, 128),
    ([129], [129], 2, 64, 128),
    ([700, 1, 255], [1000, 256, 511], 2, 128, 256),
    ([257, 3], [300, 258], 1, 64, 256),
    ([1] * 70, list(range(1, 71)), 1, 64, 16),                 # more sequences than a wave reads at once
    ([0, 0, 3] * 50 + [80], [4, 7, 40] * 50 + [81], 1, 64, 16),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case", WRITES, ids=lambda c: f"{c[0][:4]}of{c[1][:4]}x{len(c[0])}-{c[2]}x{c[3]}-b{c[4]}")
def test_writes(case, kind):
    new, kv, H, d, bt = case
    gen = torch.Generator().manual_seed(21)
    table, blocks = tables(gen, kv, bt)
    c = CodeCache(gen, kind, H, d, bt, table, blocks)
    k, v = _rows(gen, sum(new), H, d, stride_heads=len(new) % 2)
    print(f"[codes] {kind} {case[2:]}", flush=True)
    la.la_kv_write(c.layer(), k, v, _i32(_offsets(new)), _i32(kv))
    torch.cuda.synchronize()
    c.write(k, v, _offsets(new), kv)
    c.same(str(case))
    assert int(c.err) == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bt,d", [(16, 128), (64, 64), (256, 128)])
def test_blocks_filled_token_by_token(kind, bt, d):
    """Growing scales move what is there: 40 calls of one token each, two sequences, then one call that begins inside."""
    gen = torch.Generator().manual_seed(22)
    table, blocks = tables(gen, [70, 70], bt)
    c = CodeCache(gen, kind, 2, d, bt, table, blocks, filled=False)
    for half in (0, 1):                                          # the second sequence's blocks hold zeros and no scale
        code, scale = c.numbers(half)
        c.put(half, np.zeros_like(code), np.zeros_like(scale))
    c.dev.copy_(c.bytes)
    for t in range(1, 41):
        k, v = _rows(gen, 2, 2, d, spread=6.0)
        la.la_kv_write(c.layer(), k, v, _i32([0, 1, 2]), _i32([t, t + 20]))
        c.write(k, v, [0, 1, 2], [t, t + 20])
    k, v = _rows(gen, 17, 2, d, spread=9.0)
    la.la_kv_write(c.layer(), k, v, _i32([0, 9, 17]), _i32([49, 68]))
    c.write(k, v, [0, 9, 17], [49, 68])
    torch.cuda.synchronize()
    c.same(f"{kind} {bt}")


@pytest.mark.parametrize("kind", KINDS)
def test_scales_that_no_write_left(kind):
    """Inside a block whose scale is NaN, infinite, negative, zero or of too many bits, a write begins at the least."""
    gen = torch.Generator().manual_seed(23)
    table = np.arange(6, dtype=np.int32)[:, None]
    c = CodeCache(gen, kind, 1, 64, 16, table, 6)
    for half in (0, 1):
        code, scale = c.numbers(half)
        scale[:, 0] = [np.nan, np.inf, -1.0, 0.0, np.float32(1.00000012), 2.0 ** -120]
        c.put(half, code, scale)
    c.dev.copy_(c.bytes)
    k, v = _rows(gen, 6, 1, 64)
    la.la_kv_write(c.layer(), k, v, _i32(range(7)), _i32([9] * 6))
    c.write(k, v, range(7), [9] * 6)
    torch.cuda.synchronize()
    c.same(kind)


@pytest.mark.parametrize("bt", [16, 256])
@pytest.mark.parametrize("kind", KINDS)
def test_infinities_nan_zeros_and_tiny_values(kind, bt):
    gen = torch.Generator().manual_seed(24)
    table, blocks = tables(gen, [60] * 8, bt)
    c = CodeCache(gen, kind, 2, 128, bt, table, blocks)
    k, v = _rows(gen, 8 * 20, 2, 128)
    k[3, 0, 5], k[4, 1, 7], v[25, 0, 0] = float("inf"), -float("inf"), float("nan")
    k[45, :, :], v[41:60] = float("nan"), 0.0
    k[60:80] *= 2.0 ** -120
    k[80:100, 0] *= 2.0 ** 122
    v[100:120, 1] = 3.3e38
    v[120:140] = 2.0 ** -133
    cu, kv = _offsets([20] * 8), [20, 20, 50, 50, 50, 20, 33, 33]
    la.la_kv_write(c.layer(), k, v, _i32(cu), _i32(kv))
    torch.cuda.synchronize()
    c.write(k, v, cu, kv)
    c.same(kind)
    assert (int(c.err) > 0) == (kind == "int8")                  # NaN


@pytest.mark.parametrize("kind", KINDS)
def test_positions_without_a_block(kind):
    """Entries that are none, positions below zero and past the table: counted, the others written."""
    gen = torch.Generator().manual_seed(25)
    table, blocks = tables(gen, [64, 64, 64], 16)
    table[0, 1], table[1, 0] = -1, blocks + 7
    c = CodeCache(gen, kind, 2, 64, 16, table, blocks)
    new, kv = [50, 30, 20], [60, 40, 12]                         # the third's first 8 are below zero
    k, v = _rows(gen, 100, 2, 64)
    la.la_kv_write(c.layer(), k, v, _i32(_offsets(new)), _i32(kv))
    c.write(k, v, _offsets(new), kv)
    torch.cuda.synchronize()
    c.same(kind)
    assert int(c.err) >= 3
    before = int(c.err)
    la.la_kv_write(c.layer(), k, v, _i32([0, 100, 100, 100]), _i32([150, 0, 0]))
    c.write(k, v, [0, 100, 100, 100], [150, 0, 0])
    torch.cuda.synchronize()
    c.same("past the table")
    assert int(c.err) > before


@pytest.mark.parametrize("kind", KINDS)
def test_rows_outside_every_sequence(kind):
    gen = torch.Generator().manual_seed(26)
    table, blocks = tables(gen, [40, 90], 16)
    c = CodeCache(gen, kind, 2, 128, 16, table, blocks)
    k, v = _rows(gen, 60, 2, 128)
    cu, kv = [7, 20, 51], [40, 90]
    la.la_kv_write(c.layer(), k, v, _i32(cu), _i32(kv))
    c.write(k, v, cu, kv)
    torch.cuda.synchronize()
    c.same(kind)


@pytest.mark.parametrize("kind", KINDS)
def test_forks_take_their_scales_along(kind):
    """Blocks copied as bytes: the child goes on under the parent's scale, the parent keeps its own."""
    gen = torch.Generator().manual_seed(27)
    c = CodeCache(gen, kind, 2, 64, 16, np.array([[0], [1]]), 4)
    c.dev[1] = c.dev[0]
    c.bytes[1] = c.bytes[0]
    k, v = _rows(gen, 1, 2, 64)
    k, v = k * 64, v * 64
    la.la_kv_write(c.layer(slice(1, 2)), k, v, _i32([0, 1]), _i32([9]))
    keep = c.table
    c.table = keep[1:2]
    c.write(k, v, [0, 1], [9])
    torch.cuda.synchronize()
    c.same(kind)


def test_another_stream_and_a_captured_write():
    """Replays with new lengths and values write what eager calls would."""
    gen = torch.Generator().manual_seed(28)
    table, blocks = tables(gen, [80] * 3, 16)
    c = CodeCache(gen, "int8", 2, 128, 16, table, blocks)
    k, v = _rows(gen, 3, 2, 128)
    cu, kv, layer = _i32([0, 1, 2, 3]), _i32([17, 5, 70]), c.layer()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        la.la_kv_write(layer, k, v, cu, kv)
    c.write(k, v, range(4), [17, 5, 70])
    torch.cuda.synchronize()
    c.same("stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        la.la_kv_write(layer, k, v, cu, kv)
    for step in range(4):
        kn, vn = _rows(gen, 3, 2, 128, spread=8.0)
        k.copy_(kn)
        v.copy_(vn)
        kv += 1
        graph.replay()
        torch.cuda.synchronize()
        c.write(kn, vn, range(4), kv.tolist())
        c.same(f"replay {step}")


@pytest.mark.parametrize("kind", KINDS)
def test_many_short_and_empty_sequences(kind):
    """1,200 of them, most of them empty, the others of 1 to 3 tokens: written, and read back by rows of 8 and of 64 lanes."""
    gen = torch.Generator().manual_seed(29)
    new = torch.randint(-4, 4, (1200,), generator=gen).clamp(min=0).tolist()
    kv = [n + int(x) for n, x in zip(new, torch.randint(0, 20, (1200,), generator=gen))]
    for H, d in ((1, 64), (5, 128)):
        table, blocks = tables(gen, kv, 16)
        c = CodeCache(gen, kind, H, d, 16, table, blocks, layers=1, filled=False)
        k, v = _rows(gen, sum(new), H, d)
        cu = _offsets_fast(new)
        la.la_kv_write(c.layer(), k, v, cu, _i32(kv))
        c.write(k, v, cu.tolist(), kv)
        yk, yv = torch.empty_like(k, dtype=torch.float32), torch.empty_like(v, dtype=torch.float32)
        la.la_kv_read(c.layer(), yk, yv, cu, _i32(kv))
        torch.cuda.synchronize()
        c.same(kind)
        assert int(c.err) == 0
        for half, y in ((0, yk), (1, yv)):
            code, scale = c.numbers(half)
            seq = np.repeat(np.arange(1200), new)
            pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, kv)])
            block = table[seq, pos // 16]
            assert np.array_equal(y.double().cpu().numpy(), code[block, :, pos % 16] * scale[block][..., None])


def _offsets_fast(new):
    return torch.cumsum(torch.tensor([0] + new), 0).to(torch.int32).cuda()


@pytest.mark.parametrize("kind", KINDS)
def test_offsets_past_the_rows(kind):
    """Tokens that cu_seqlens has and the call's rows have not are not written; the others are where they belong."""
    gen = torch.Generator().manual_seed(30)
    table, blocks = tables(gen, [70, 50], 16)
    c = CodeCache(gen, kind, 2, 64, 16, table, blocks)
    k, v = _rows(gen, 40, 2, 64)
    la.la_kv_write(c.layer(), k[:30].contiguous(), v[:30].contiguous(), _i32([0, 20, 40]), _i32([65, 50]))
    c.write(k, v, [0, 20], [65])
    keep, c.table = c.table, c.table[1:]
    c.write(k, v, [20, 30], [40])                                # the second's first ten: keys 30 to 39
    c.table = keep
    torch.cuda.synchronize()
    c.same(kind)


# --- reads -----------------------------------------------------------------------

READS = [([1], [1], 1, 64, 16), ([5, 0, 40, 16], [21, 9, 57, 16], 2, 128, 16), ([100, 33], [131, 33], 3, 64, 32),
         ([300, 2], [700, 256], 2, 128, 256)]


def _round(x, out):
    return torch.from_numpy(x).to(out.dtype) if out.dtype is torch.float32 else torch.from_numpy(x).float().to(out.dtype)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case", READS, ids=str)
def test_reads_of_codes(case, kind, out):
    new, kv, H, d, bt = case
    gen = torch.Generator().manual_seed(31)
    table, blocks = tables(gen, kv, bt)
    c = CodeCache(gen, kind, H, d, bt, table, blocks)
    T = sum(new)
    wide = torch.full((T + 6, 2 * H + 1, d), 9.0, dtype=out, device="cuda")      # rows before and behind, a column between
    k, v = wide[:, :H], wide[:, H:2 * H]
    la.la_kv_read(c.layer(), k, v, _i32(_offsets(new, 2)), _i32(kv))
    torch.cuda.synchronize()
    for half, y in ((0, k), (1, v)):
        want = np.concatenate([c.rows(i, L, half)[L - n:] for i, (n, L) in enumerate(zip(new, kv))])
        assert torch.equal(y[2:2 + T].cpu(), _round(want, y)), half
    rest = torch.cat([wide[:2].flatten(), wide[2 + T:].flatten(), wide[:, 2 * H:].flatten()])
    assert (rest == 9.0).all() and int(c.err) == 0


@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("fp8", "bf16"), ("fp8", "f32")])
def test_reads_of_other_caches(kind, out):
    """What la_kv_write put there comes back."""
    store = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}[kind]
    io = torch.float32 if kind == "f32" else torch.bfloat16
    ks, vs = (0.37, 0.11) if kind == "fp8" else (1.0, 1.0)
    gen = torch.Generator().manual_seed(32)
    new, kv, H, d, bt = [40, 0, 3], [57, 3, 19], 3, 128, 16
    table, blocks = tables(gen, kv, bt)
    size = 2 * H * bt * d * torch.empty(0, dtype=store).element_size()
    cache = torch.zeros((blocks, size), dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    layer = la.make_kv_layer(cache, torch.from_numpy(table).cuda(), bt, H, d, store, k_scale=ks, v_scale=vs, err_count=err)
    k, v = (torch.randn((sum(new), H, d), generator=gen).to(io).cuda() for _ in (0, 1))
    la.la_kv_write(layer, k, v, _i32(_offsets(new)), _i32(kv))
    dt = torch.float32 if out == "f32" else torch.bfloat16
    yk, yv = torch.empty(k.shape, dtype=dt, device="cuda"), torch.empty(k.shape, dtype=dt, device="cuda")
    la.la_kv_read(layer, yk, yv, _i32(_offsets(new)), _i32(kv))
    torch.cuda.synchronize()
    for x, y, s in ((k, yk, ks), (v, yv, vs)):
        if kind == "fp8":
            s = np.float32(s)
            code = kc.e4m3(np.clip((x.float().cpu().numpy() / s).astype(np.float64), -448, 448))
            want = torch.from_numpy((code * np.float64(s)).astype(np.float32)).to(dt)
        else:
            want = x.to(dt).cpu()
        assert torch.equal(y.cpu(), want)
    assert int(err) == 0


@pytest.mark.parametrize("kind", KINDS)
def test_reads_without_a_block(kind):
    gen = torch.Generator().manual_seed(33)
    table, blocks = tables(gen, [64, 64], 16)
    table[0, 1] = -1
    c = CodeCache(gen, kind, 2, 64, 16, table, blocks)
    new, kv = [64, 20], [64, 12]
    k, v = (torch.full((84, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in (0, 1))
    la.la_kv_read(c.layer(), k, v, _i32(_offsets(new)), _i32(kv))
    torch.cuda.synchronize()
    for half, y in ((0, k), (1, v)):
        want = np.concatenate([c.rows(0, 64, half), np.zeros((8, 2, 64)), c.rows(1, 12, half)])
        assert torch.equal(y.cpu(), _round(want, y))
    assert int(c.err) >= 24


@pytest.mark.parametrize("kind", KINDS)
def test_blocks_past_four_gigabytes(kind):
    """The last blocks of a cache of 5 GiB."""
    gen = torch.Generator().manual_seed(34)
    H, d, bt, blocks = 2, 128, 16, 5 * 2 ** 30 // 65536
    layer_bytes = 2 * H * bt * d
    cache = torch.zeros((blocks, 65536), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[blocks - 1, blocks - 2]], dtype=torch.int32, device="cuda")
    layer = la.make_kv_layer(cache, table, bt, H, d, TYPES[kind], k_offset=65536 - 2 * layer_bytes, k_scales=64)
    k, v = _rows(gen, 20, H, d)
    la.la_kv_write(layer, k, v, _i32([0, 20]), _i32([20]))
    yk, yv = torch.empty_like(k, dtype=torch.float32), torch.empty_like(v, dtype=torch.float32)
    la.la_kv_read(layer, yk, yv, _i32([0, 20]), _i32([20]))
    torch.cuda.synchronize()
    small = CodeCache(gen, kind, H, d, bt, np.array([[0, 1]]), 2)
    small.write(k, v, [0, 20], [20])
    for half, y in ((0, yk), (1, yv)):
        assert np.array_equal(y.double().cpu().numpy(), small.rows(0, 20, half))
