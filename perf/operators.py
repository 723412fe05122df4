"""Performance cases of the attention side of a hybrid cache: attention of whole
prompts and of resumed suffixes, attention of generated tokens over a cache
whose requests share prefixes, the writing of new keys and values into cache
blocks, and the cache blocks' own bookkeeping (fork, free, extend, compact).

`listed()` holds the fixed cases, `draw(rng)` one more of the same ranges,
`prepare` what an engine has in hand before the call, `run` one pass (plain
torch in 32 bits, or the library's entry points where `own` is set), `work`
what a pass cannot do without and `exact` the same outputs in 64 bits.

Queries, keys and values are normal; some channels of the keys are strong, so
that the scores of a row spread over several units, as trained ones do.
"""
from __future__ import annotations

import math
import random

import torch

own = False        # True: run() calls the library

DEV = "cuda"
LAYERS = 4         # attention layers that share a cache block; the cases use the second one
F8_MAX = 448.0     # largest finite value of the 8-bit cache type

# The 16-sequence batch: prompt lengths and the boundaries its cached prefixes allow (0: nothing cached).
VARLEN_N = [7760, 8016, 5376, 8064, 3136, 4000, 2656, 5136, 6080, 6320, 4096, 1216, 3696, 7152, 1968, 2784]
VARLEN_B = [0, 7936, 1536, 0, 0, 0, 1024, 0, 0, 6144, 0, 256, 3328, 6912, 1792, 1280]


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")] if text else []


def _prompt(name, new, heads, kv_heads, dim, dtype="bf16", kv="", store="packed", cache="", block=16, fused=False):
    """new: tokens each sequence computes; kv: its length with what the cache
    holds before them (empty: nothing); store: keys and values packed beside
    the queries, or in cache blocks; fused: q, k, v are slices of one tensor."""
    return {"name": name, "kind": "prompt", "new": _text(new), "kv": _text(kv) if kv else "", "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "store": store, "cache": cache or dtype, "block": block,
            "fused": fused}


def _decode(name, kv, heads, kv_heads, dim, dtype="bf16", cache="", block=16, groups="", prefix=""):
    """kv: every sequence's length with its new token; groups: sizes of the
    consecutive groups that share a prefix of `prefix` tokens (empty: none)."""
    return {"name": name, "kind": "decode", "kv": _text(kv), "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "cache": cache or dtype, "block": block, "groups": _text(groups) if groups else "",
            "prefix": _text(prefix) if groups else ""}


def _write(name, new, kv, kv_heads, dim, dtype="bf16", cache="", block=16):
    return {"name": name, "kind": "write", "new": _text(new), "kv": _text(kv), "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "cache": cache or dtype, "block": block}


def _fork(name, lens, beams, block=16, block_bytes=132288):
    """lens: the tokens so far of each search; beams: its candidates."""
    return {"name": name, "kind": "fork", "lens": _text(lens), "beams": beams, "block": block,
            "block_bytes": block_bytes}


def _retire(name, lens, quarter=4, block=16, block_bytes=132288):
    return {"name": name, "kind": "retire", "lens": _text(lens), "quarter": quarter, "block": block,
            "block_bytes": block_bytes}


def _spread(seed, n, lo, hi):
    """n lengths between lo and hi, even over their logarithm."""
    r = random.Random(seed)
    return [_log_int(r, lo, hi) for _ in range(n)]


def listed():
    return [
        # The shortest prompt of the serial sweep: few rows, where latency counts.
        _prompt("prompt_512_h8", [512], 8, 2, 128),
        # The longest prompt the model takes.
        _prompt("prompt_32768_h16", [32768], 16, 4, 128, fused=True),
        # fp32, the accuracy path: three ragged prompts at the small head size, a key head for each query head.
        _prompt("prompt_f32_ragged3", [1791, 640, 257], 8, 8, 64, "f32"),
        # A reloaded prompt's strict-prefix suffix over its restored blocks.
        _prompt("resume_256_at_3328_h8", [256], 8, 2, 128, kv=[3584], store="paged"),
        # A mixed batch over an 8-bit cache: cold prompts, full and partial prefix hits in one call.
        _prompt("resume_varlen16_fp8", [n - b for n, b in zip(VARLEN_N, VARLEN_B)], 8, 2, 128, kv=VARLEN_N,
                store="paged", cache="fp8"),
        # One generated token of one request: the smallest attention call there is.
        _decode("decode_1seq_3584_h8", [3584], 8, 2, 128),
        # A full serving batch under one long system prompt, with answers of all lengths.
        _decode("decode_64seq_shared_6144", [6144 + n for n in _spread(3, 64, 1, 1500)], 16, 4, 128, groups=[64],
                prefix=[6144]),
        # Unrelated requests of every age over an 8-bit cache, one of them at the longest context.
        _decode("decode_96seq_ragged_fp8", [32768, 1] + _spread(4, 94, 17, 20000), 16, 4, 128, cache="fp8"),
        # The new token of each of 64 requests goes into its block.
        _write("write_64tokens", [1] * 64, _spread(5, 64, 1, 8000), 8, 128),
        # The suffixes of the mixed batch go into 8-bit blocks.
        _write("write_varlen16_fp8", [n - b for n, b in zip(VARLEN_N, VARLEN_B)], VARLEN_N, 8, 128, cache="fp8"),
        # A step of eight searches of eight candidates: each forks one of the last step's, and those are freed.
        _fork("fork_8x8_3584", [3583, 3584, 1001, 2050, 517, 3333, 2719, 3001], 8),
        # A quarter of the requests end, the cache is compacted, as many new ones come in.
        _retire("retire_16x3328", [3328, 3300, 2500, 1000, 3328, 1600, 2999, 3328, 3000, 2048, 3328, 17, 1500, 3328,
                                   800, 3001]),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cut(rng, total, most, n):
    """n ragged lengths of about `total` tokens, each at most `most`."""
    w = [rng.random() + 0.02 for _ in range(n)]
    return [min(most, max(1, int(total * x / sum(w)))) for x in w]


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "resume", "resume", "decode", "decode", "shared", "write", "fork", "retire"])
    dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
    kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 4), (8, 1), (3, 2), (2, 16), (5, 1), (4, 7)])
    dim, block = rng.choice([64, 128, 128]), rng.choice([16, 16, 16, 32, 64, 128])
    heads = kv_heads * group
    if kind in ("prompt", "resume"):
        # a call costs by its tokens times the keys before them times its heads: both are kept below the listed ones'
        total = _log_int(rng, 16, 2048 if dtype == "f32" else 16384)
        new = _cut(rng, total, 12000, rng.randint(1, max(1, min(24, total // 24))))
        if kind == "prompt":
            c = _prompt("", new, heads, kv_heads, dim, dtype, fused=rng.random() < 0.5)
        else:
            c = _prompt("", new, heads, kv_heads, dim, dtype, [n + _log_int(rng, 1, 4096) for n in new], "paged", cache,
                        block)
    elif kind == "decode":
        n = _log_int(rng, 1, 128)
        c = _decode("", [_log_int(rng, 1, 16000 if n < 48 else 6000) for _ in range(n)], heads, kv_heads, dim, dtype,
                    cache, block)
    elif kind == "shared":
        groups = [_log_int(rng, 1, 64) for _ in range(rng.randint(1, 4))]
        prefix = [block * _log_int(rng, 1, 8192 // block) for _ in groups]
        kv = [p + _log_int(rng, 1, 1024) for g, p in zip(groups, prefix) for _ in range(g)]
        c = _decode("", kv, heads, kv_heads, dim, dtype, cache, block, groups, prefix)
    elif kind == "write":
        new = _cut(rng, _log_int(rng, 16, 49152), 8192, rng.randint(1, 64))
        c = _write("", new, [n + rng.randint(0, 2000) for n in new], kv_heads, dim, dtype, cache, block)
    elif kind == "fork":
        c = _fork("", [_log_int(rng, 1, 4096) for _ in range(rng.randint(1, 12))], rng.randint(1, 8), block,
                  rng.choice([16384, 65536, 132288]))
    else:
        quarter = rng.randint(1, 6)
        c = _retire("", [_log_int(rng, 1, 3328) for _ in range(4 * quarter)], quarter, block,
                    rng.choice([16384, 65536, 132288]))
    c.pop("name", None)
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (2 ** 31) + 23)
    return g


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}[name]


def _size(name):
    return {"bf16": 2, "f32": 4, "fp8": 1}[name]


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device=DEV)


def _offsets(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def _up(a, b):
    return -(-a // b)


def _kv_scales(case):
    """What a stored value stands for, per unit: the 8-bit cache's scales, as a calibration would give them."""
    return (0.0625, 0.03125) if case["cache"] == "fp8" else (1.0, 1.0)


def _keys(gen, shape):
    """Keys with a few strong channels."""
    k = torch.randn(shape, generator=gen, device=DEV)
    return k * (1.0 + 4.0 * (torch.arange(shape[-1], device=DEV) % 16 == 3))


def _cache(case, gen, blocks):
    """A cache of `blocks` blocks, each with the keys and values of LAYERS
    layers, the used one filled; bytes [blocks, block_bytes]."""
    H, bt, d = case["kv_heads"], case["block"], case["dim"]
    part = H * bt * d * _size(case["cache"])
    cache = torch.zeros((blocks, 2 * part * LAYERS), dtype=torch.uint8, device=DEV)
    ks, vs = _kv_scales(case)
    for half, scale, x in ((0, ks, _keys(gen, (blocks, H, bt, d))),
                           (1, vs, torch.randn((blocks, H, bt, d), generator=gen, device=DEV))):
        _part(case, cache, half).copy_((x / scale).to(_type(case["cache"])))
    return cache


def _part(case, cache, half):
    """The used layer's keys (0) or values (1) in the cache: [blocks, kv heads, block tokens, dim]."""
    H, bt, d = case["kv_heads"], case["block"], case["dim"]
    t = _type(case["cache"])
    part = H * bt * d * _size(case["cache"])
    at = (2 + half) * part
    return cache[:, at:at + part].view(t).unflatten(1, (H, bt, d))


def _tables(case, kv, gen, shared=()):
    """Block tables [sequences, most blocks] over a permuted cache, -1 behind
    each sequence's last block; shared: (first sequence, sequences, tokens)
    whose leading whole blocks are one set."""
    bt = case["block"]
    need = torch.tensor([_up(n, bt) for n in kv], device=DEV)
    most = int(need.max())
    slot = torch.arange(most, device=DEV)[None, :]
    perm = torch.randperm(int(need.sum()) + 7, generator=gen, device=DEV)
    first = torch.cumsum(need, 0) - need
    table = torch.where(slot < need[:, None], perm[(first[:, None] + slot).clamp(max=len(perm) - 1)], -1)
    for at, n, tokens in shared:
        table[at:at + n, :tokens // bt] = table[at, :tokens // bt]
    return table.to(torch.int32).contiguous(), len(perm)


def prepare(case, seed):
    gen = _gen(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("fork", "retire"):
        return _prepare_blocks(case, gen, s)
    td, d, H = _type(case["dtype"]), case["dim"], case["kv_heads"]
    if kind == "prompt":
        new, Hq = _ints(case["new"]), case["heads"]
        kv = _ints(case["kv"]) or new
        T = sum(new)
        if case["store"] == "packed":
            x = torch.randn((T, Hq + 2 * H, d), generator=gen, device=DEV)
            x[:, Hq:Hq + H] = _keys(gen, (T, H, d))
            x = x.to(td)
            parts = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
            s["q"], s["k"], s["v"] = parts if case["fused"] else (p.contiguous() for p in parts)
        else:
            s["q"] = torch.randn((T, Hq, d), generator=gen, device=DEV).to(td)
            s["table"], blocks = _tables(case, kv, gen)
            s["cache"] = _cache(case, gen, blocks)
        s["new"], s["kv"], s["cu"], s["kv_dev"] = new, kv, _i32(_offsets(new)), _i32(kv)
        return s
    kv = _ints(case["kv"])
    if kind == "decode":
        groups, prefix = _ints(case["groups"]), _ints(case["prefix"])
        shared = list(zip(_offsets(groups), groups, prefix))
        s["q"] = torch.randn((len(kv), case["heads"], d), generator=gen, device=DEV).to(td)
        s["table"], blocks = _tables(case, kv, gen, shared)
        s["cache"] = _cache(case, gen, blocks)
        s["kv"], s["kv_dev"] = kv, _i32(kv)
        s["cu_group"], s["prefix"] = _i32(_offsets(groups)), _i32(prefix)
        return s
    new = _ints(case["new"])
    T = sum(new)
    s["k"], s["v"] = _keys(gen, (T, H, d)).to(td), torch.randn((T, H, d), generator=gen, device=DEV).to(td)
    s["table"], blocks = _tables(case, kv, gen)
    s["cache"] = _cache(case, gen, blocks)
    s["new"], s["kv"], s["cu"], s["kv_dev"] = new, kv, _i32(_offsets(new)), _i32(kv)
    return s


def _prepare_blocks(case, gen, s):
    """A pool of blocks with its tables, counts and stack of free blocks.  fork:
    a row for each candidate of every search (its search's whole blocks and a
    last one of its own) and as many empty rows.  retire: every row holds a
    request; the last quarter came in last, above the others."""
    bt, lens = case["block"], _ints(case["lens"])
    if case["kind"] == "fork":
        beams, n = case["beams"], len(lens) * case["beams"]
        search = torch.arange(n, device=DEV) // beams
        whole = torch.tensor([x // bt for x in lens], device=DEV)
        tail = torch.tensor([x % bt > 0 for x in lens], device=DEV)[search]
        used = int(whole.sum()) + int(tail.sum())
        blocks, width = used + 2 * n + 5, max(lens) // bt + 1
        perm = torch.randperm(used, generator=gen, device=DEV).to(torch.int32)
        slot = torch.arange(width, device=DEV)[None, :]
        first = (torch.cumsum(whole, 0) - whole)[search][:, None]
        own_at = (int(whole.sum()) + torch.cumsum(tail, 0) - 1)[:, None]
        end = whole[search][:, None]
        rows = torch.where(slot < end, perm[(first + slot).clamp(max=used - 1)],
                           torch.where((slot == end) & tail[:, None], perm[own_at.clamp(min=0)], -1))
        s["table"] = torch.cat([rows, torch.full_like(rows, -1)]).to(torch.int32).contiguous()
        parent = search * beams + torch.randint(0, beams, (n,), generator=gen, device=DEV)
        s["rows"] = (_i32(range(n)), _i32(range(n, 2 * n)))
        s["parents"] = (parent.to(torch.int32), (parent + n).to(torch.int32))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)[search].contiguous()
    else:
        n, k = len(lens), case["quarter"]
        need = [_up(x, bt) for x in lens]
        used, width = sum(need), max(need) + 1
        blocks = used + 5
        low = sum(need[:n - k])
        perm = torch.cat([torch.randperm(low, generator=gen, device=DEV), torch.arange(low, used, device=DEV)])
        first, nd = torch.tensor(_offsets(need)[:n], device=DEV)[:, None], torch.tensor(need, device=DEV)[:, None]
        slot = torch.arange(width, device=DEV)[None, :]
        s["table"] = torch.where(slot < nd, perm[(first + slot).clamp(max=used - 1)], -1).to(torch.int32).contiguous()
        # quarters retire in turn, so that the newest one always stays: 0, 1, 2, 3, 0, ...
        s["rows"] = tuple(_i32(range(a, a + k)) for a in range(0, n, k))
        s["lens"] = tuple(_i32(lens[a:a + k]) for a in range(0, n, k))
    s["ref"] = torch.bincount(s["table"][s["table"] >= 0], minlength=blocks).to(torch.int32)
    s["free"] = torch.zeros(blocks, dtype=torch.int32, device=DEV)
    s["free"][:blocks - used] = torch.arange(blocks - 1, used - 1, -1, dtype=torch.int32, device=DEV)
    s["free_count"] = _i32([blocks - used])
    s["cache"] = torch.randint(0, 256, (blocks, case["block_bytes"]), generator=gen, device=DEV, dtype=torch.uint8)
    s["step"] = 0
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    s, kind = state, state["case"]["kind"]
    if kind in ("fork", "retire"):
        return _run_blocks(s)
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2609_15030_amd import api
    from paper_2609_15030_amd import linattn as la
    c = s["case"]
    ks, vs = _kv_scales(c)
    if "cache" in s and "layer" not in s:
        part = c["kv_heads"] * c["block"] * c["dim"] * _size(c["cache"])
        s["layer"] = la.make_kv_layer(s["cache"], s["table"], c["block"], c["kv_heads"], c["dim"], _type(c["cache"]),
                                      k_offset=2 * part, v_offset=3 * part, k_scale=ks, v_scale=vs)
    if c["kind"] == "prompt":
        if "plan" not in s:      # lengths, workspace: what a program keeps
            s["plan"] = api.AttnPrefill(c["heads"], c["kv_heads"], c["dim"], s["new"],
                                        s["kv"] if c["store"] == "paged" else None, _type(c["dtype"]))
        return [s["plan"].run(s["q"], s["k"], s["v"]) if c["store"] == "packed" else s["plan"].run_paged(s["layer"], s["q"])]
    if c["kind"] == "decode":
        if "plan" not in s:
            s["plan"] = api.AttnDecode(len(s["kv"]), c["heads"], c["kv_heads"], c["dim"], max(s["kv"]),
                                       _type(c["dtype"]), cu_group=s["cu_group"] if c["groups"] else None,
                                       max_prefix_len=max(_ints(c["prefix"]) or [0]))
        return [s["plan"].run(s["layer"], s["q"], s["kv_dev"], s["prefix"] if c["groups"] else None)]
    la.la_kv_write(s["layer"], s["k"], s["v"], s["cu"], s["kv_dev"])
    return [_part(c, s["cache"], 0), _part(c, s["cache"], 1)]


def _gather(s, half, most):
    """Cached keys or values of every sequence: [sequences, most, kv heads, dim] in 32 bits."""
    c = s["case"]
    x = _part(c, s["cache"], half)[s["table"].long().clamp(min=0)].float() * _kv_scales(c)[half]
    return x.transpose(2, 3).flatten(1, 2)[:, :most]


def _pad(x, cu, most):
    """Packed rows as [sequences, most, ...], zeros behind each sequence's end."""
    at = torch.arange(most, device=DEV)[None, :]
    n = (cu[1:] - cu[:-1])[:, None]
    rows = (cu[:-1, None] + at).clamp(max=x.shape[0] - 1)
    return x.float()[rows.long()] * (at < n).reshape(n.shape[0], most, *[1] * (x.dim() - 1))


def _attend(q, k, v, pos, kv_len, scale):
    """softmax(scale q k^T) v over the keys j <= pos, j < kv_len, in 32 bits;
    q [n, rows, heads, d], k, v [n, keys, kv heads, d], pos [n, rows]."""
    n, rows, heads, d = q.shape
    keys, H = k.shape[1], k.shape[2]
    kt = k.permute(0, 2, 3, 1).contiguous()
    vv = v.transpose(1, 2).contiguous()
    out = torch.empty_like(q)
    step = max(1, 2 ** 31 // max(1, n * heads * keys))      # rows at a time, so that their scores fit in memory
    for a in range(0, rows, step):
        b = min(rows, a + step)
        x = q[:, a:b].reshape(n, b - a, H, heads // H, d).permute(0, 2, 3, 1, 4).reshape(n, H, -1, d)
        seen = torch.minimum(pos[:, a:b] + 1, kv_len[:, None])[:, None, None, :, None] > torch.arange(keys, device=DEV)
        p = (x @ kt).mul_(scale).reshape(n, H, heads // H, b - a, keys)
        p.masked_fill_(~seen, -math.inf)
        m = p.amax(-1, keepdim=True)
        p.sub_(m.masked_fill(m == -math.inf, 0.0)).exp_()
        total = p.sum(-1, keepdim=True)
        o = (p.reshape(n, H, -1, keys) @ vv).reshape(n, H, heads // H, b - a, d) / total.masked_fill(total == 0, 1.0)
        out[:, a:b] = o.permute(0, 3, 1, 2, 4).reshape(n, b - a, heads, d)
    return out


def _run_plain(s):
    c = s["case"]
    kv_len = s["kv_dev"]
    most = max(s["kv"])
    scale = c["dim"] ** -0.5
    if c["kind"] == "decode":
        o = _attend(s["q"].float()[:, None], _gather(s, 0, most), _gather(s, 1, most), kv_len[:, None] - 1, kv_len, scale)
        return [o[:, 0].to(s["q"].dtype)]
    cu = s["cu"]
    n = (cu[1:] - cu[:-1])[:, None]
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEV), n[:, 0].long(), output_size=sum(s["new"]))
    local = torch.arange(sum(s["new"]), device=DEV) - cu[seq]
    if c["kind"] == "write":
        pos = local + (kv_len - n[:, 0])[seq]
        block = s["table"][seq, pos // c["block"]].long()
        for half, x in ((0, s["k"]), (1, s["v"])):
            y = x.float() / _kv_scales(c)[half]
            if c["cache"] == "fp8":
                y = y.clamp(-F8_MAX, F8_MAX)
            to = _part(c, s["cache"], half)
            same = torch.uint8 if c["cache"] == "fp8" else to.dtype        # the 8-bit type takes no indexed store
            to.view(same)[block, :, pos % c["block"]] = y.to(to.dtype).view(same)
        return [_part(c, s["cache"], 0), _part(c, s["cache"], 1)]
    rows = max(s["new"])
    if c["store"] == "packed":
        k, v = _pad(s["k"], cu, rows), _pad(s["v"], cu, rows)
    else:
        k, v = _gather(s, 0, most), _gather(s, 1, most)
    pos = torch.arange(rows, device=DEV)[None, :] + (kv_len[:, None] - n)
    o = _attend(_pad(s["q"], cu, rows), k, v, pos, kv_len, scale)
    return [o[seq, local].to(s["q"].dtype)]


def _run_blocks(s):
    """fork: the next candidates fork the last ones, which are then freed; the
    halves of the table take turns.  retire: a quarter of the requests end,
    the cache is compacted and as many new requests get their blocks."""
    c, step = s["case"], s["step"]
    s["step"] = step + 1
    if own and "pool" not in s:
        from paper_2609_15030_amd import api
        s["pool"] = api.BlockPool(s["cache"], c["block"], s["table"], s["ref"], s["free"], s["free_count"])
    p = s["pool"] if own else _PlainPool(s)
    if c["kind"] == "fork":
        old, new = s["rows"][step % 2], s["rows"][(step + 1) % 2]
        p.fork(s["parents"][step % 2], new, s["lens"])
        p.free(old)
    else:
        k = step % len(s["rows"])
        p.free(s["rows"][k])
        p.compact()
        p.extend(s["rows"][k], s["lens"][k])
    return [s["table"], s["ref"], s["free_count"], s["free"], s["cache"]]


class _PlainPool:
    """The block operations in plain torch, on the state's tensors."""

    def __init__(self, s):
        self.s, self.bt = s, s["case"]["block"]
        self.width, self.blocks = s["table"].shape[1], s["ref"].shape[0]

    def _take(self, want):
        """The fresh blocks for the marked places, in order, with one reference each."""
        s = self.s
        rank = torch.cumsum(want.reshape(-1), 0).reshape(want.shape) - 1
        ids = s["free"][(s["free_count"] - 1 - rank).clamp(min=0).long()]
        s["ref"].index_put_((ids[want].long(),), torch.ones_like(ids[want]))
        s["free_count"] -= want.sum().to(torch.int32)
        return ids

    def fork(self, parent, child, lens):
        s = self.s
        full, rest = lens // self.bt, lens % self.bt > 0
        slot = torch.arange(self.width, device=DEV)[None, :]
        src = s["table"][parent.long()]
        keep = slot < full[:, None]
        s["ref"] += torch.bincount(src[keep], minlength=self.blocks).to(torch.int32)
        tail = self._take(rest)
        s["table"][child.long()] = torch.where(keep, src, torch.where((slot == full[:, None]) & rest[:, None], tail[:, None], -1))
        s["cache"][tail[rest].long()] = s["cache"][src.gather(1, full[:, None].long())[rest, 0].long()]

    def free(self, rows):
        s = self.s
        ids = s["table"][rows.long()]
        had = s["ref"] > 0
        s["ref"] -= torch.bincount(ids[ids >= 0], minlength=self.blocks).to(torch.int32)
        s["table"][rows.long()] = -1
        gone = torch.nonzero(had & (s["ref"] == 0))[:, 0].to(torch.int32)
        s["free"].index_copy_(0, s["free_count"].long() + torch.arange(len(gone), device=DEV), gone)
        s["free_count"] += len(gone)

    def compact(self):
        s = self.s
        live = s["ref"] > 0
        n = int(live.sum())
        ids = torch.arange(self.blocks, device=DEV)
        src, dst = ids[n:][live[n:]], ids[:n][~live[:n]]
        s["cache"][dst] = s["cache"][src]
        to = ids.clone()
        to[src] = dst
        s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()].to(torch.int32), s["table"]))
        s["ref"][dst] = s["ref"][src]
        s["ref"][n:] = 0
        s["free"][:self.blocks - n] = torch.arange(self.blocks - 1, n - 1, -1, dtype=torch.int32, device=DEV)
        s["free_count"].fill_(self.blocks - n)

    def extend(self, rows, lens):
        s = self.s
        table = s["table"][rows.long()]
        slot = torch.arange(self.width, device=DEV)[None, :]
        want = (slot < ((lens + self.bt - 1) // self.bt)[:, None]) & (table < 0)
        s["table"][rows.long()] = torch.where(want, self._take(want), table)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("fork", "retire"):
        lens, bt, size = _ints(case["lens"]), case["block"], case["block_bytes"]
        need = [_up(n, bt) for n in lens]
        if kind == "fork":       # a last block copied for each child whose parent ends inside one; entries read and written
            return {"bytes": case["beams"] * (2.0 * size * sum(n % bt > 0 for n in lens) + 16.0 * sum(need)), "flops": 0}
        k = case["quarter"]      # the newest quarter's blocks move into the holes of the one that ends
        ends = [sum(need[a:a + k]) for a in range(0, len(lens), k)]
        return {"bytes": 2.0 * size * min(ends[0], ends[-1]) + 16.0 * sum(need), "flops": 0}
    d, H, kv, e, ce = case["dim"], case["kv_heads"], _ints(case["kv"]), _size(case["dtype"]), _size(case["cache"])
    if kind == "write":
        T = sum(_ints(case["new"]))
        return {"bytes": 2.0 * T * H * d * (e + ce), "flops": 0}
    heads = case["heads"]
    if kind == "decode":
        groups, prefix = _ints(case["groups"]), _ints(case["prefix"])
        again = sum((g - 1) * p for g, p in zip(groups, prefix))       # read once for its group
        return {"bytes": 2.0 * (sum(kv) - again) * H * d * ce + 2.0 * len(kv) * heads * d * e,
                "flops": 4.0 * d * heads * sum(kv)}
    new = _ints(case["new"])
    kv = kv or new
    pairs = sum(n * (L - n) + n * (n + 1) / 2 for n, L in zip(new, kv))
    return {"bytes": 2.0 * sum(new) * heads * d * e + 2.0 * sum(kv) * H * d * ce, "flops": 4.0 * d * heads * pairs}


# ---------------------------------------------------------------------------
# 64-bit results, sequence by sequence from the definition
# ---------------------------------------------------------------------------

def _exact_rows(q, k, v, first):
    """One sequence and one query head: rows at positions first, first + 1, ... over all keys."""
    out = torch.zeros_like(q)
    step = max(1, 2 ** 28 // max(1, k.shape[0]))
    for a in range(0, q.shape[0], step):
        x = torch.mm(q[a:a + step], k.t().contiguous()) / math.sqrt(q.shape[1])
        late = torch.arange(k.shape[0], device=DEV)[None, :] > first + a + torch.arange(x.shape[0], device=DEV)[:, None]
        x[late] = -math.inf
        out[a:a + step] = torch.softmax(x, 1) @ v
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "retire"):
        return None
    s = prepare(case, seed)
    c, kv, d = case, s["kv"], case["dim"]
    ks, vs = _kv_scales(c)
    if kind == "write":
        outs = []
        for half, x, scale in ((0, s["k"], ks), (1, s["v"], vs)):
            to = _part(c, s["cache"], half).double()
            y = x.double() / scale
            y = y.clamp(-F8_MAX, F8_MAX) if c["cache"] == "fp8" else y
            at = 0
            for i, n in enumerate(s["new"]):
                pos = torch.arange(kv[i] - n, kv[i], device=DEV)
                to[s["table"][i].long()[pos // c["block"]], :, pos % c["block"]] = y[at:at + n]
                at += n
            outs.append(to)
        return outs
    G = c["heads"] // c["kv_heads"]
    new = s["new"] if kind == "prompt" else [1] * len(kv)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for i, (n, L) in enumerate(zip(new, kv)):
        if "cache" in s:
            ids = s["table"][i, :_up(L, c["block"])].long()
            k, v = (_part(c, s["cache"], h)[ids].double().transpose(1, 2).flatten(0, 1)[:L] * (ks, vs)[h] for h in (0, 1))
        else:
            k, v = s["k"][at:at + n].double(), s["v"][at:at + n].double()
        for h in range(c["heads"]):
            out[at:at + n, h] = _exact_rows(s["q"][at:at + n, h].double(), k[:, h // G].contiguous(),
                                            v[:, h // G].contiguous(), L - n)
        at += n
    return [out]
