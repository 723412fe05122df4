"""Performance cases of an attention layer whose cache holds 8 bits with a scale
for each block of tokens and key head: rotary positions of queries and keys,
the quantising write and the read of such a cache, and attention over it
(suffixes of prompts, generated tokens, shared prefixes).

`listed()` holds the fixed cases, `draw(rng)` one more of the same ranges,
`prepare` what an engine has in hand before the call, `run` one pass (plain
torch in 32 bits, or the library's entry points where `own` is set), `work`
what a pass cannot do without and `exact` the same outputs in 64 bits.

A cache block holds LAYERS layers' keys and values, [kv heads, block tokens,
dim] of 8-bit codes each, and behind them the scales, fp32 [kv heads] for each
layer's keys and values.  A code c stands for c times its block's and head's scale:

  e4m3   the smallest power of two with max |x| <= 448 scale
  int8   max |x| / 127, rounded up to 8 significant bits

over the tokens written together, and never less than what the tokens that
stay in the block had; those follow a scale that grows.

Queries, keys and values are normal; some channels of the keys are strong, so
that the scores of a row spread over several units, as trained ones do.
"""
from __future__ import annotations

import math
import random

import torch

own = False        # True: run() calls the library

DEV = "cuda"
LAYERS = 2         # attention layers that share a cache block; the cases use the second one
MOST = {"e4m3": 448.0, "int8": 127.0}      # largest code
LEAST = 2.0 ** -100                        # smallest scale

# The 16-sequence batch: prompt lengths and the boundaries its cached prefixes allow (0: nothing cached).
VARLEN_N = [7760, 8016, 5376, 8064, 3136, 4000, 2656, 5136, 6080, 6320, 4096, 1216, 3696, 7152, 1968, 2784]
VARLEN_B = [0, 7936, 1536, 0, 0, 0, 1024, 0, 0, 6144, 0, 256, 3328, 6912, 1792, 1280]
VARLEN_NEW = [n - b for n, b in zip(VARLEN_N, VARLEN_B)]


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")] if text else []


def _rope(name, new, kv, heads, kv_heads, dim, rotary, layout="halves", dtype="bf16", scaling="", scattered=False,
          fused=False, transpose=False, base=10000.0):
    """kv: every sequence's length with its new tokens; scattered: a position for
    each token instead; scaling: kind and numbers; fused: slices of one
    projection; transpose: the gradient."""
    return {"name": name, "kind": "rope", "new": _text(new), "kv": _text(kv), "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "rotary": rotary, "layout": layout, "dtype": dtype, "scaling": scaling, "scattered": scattered,
            "fused": fused, "transpose": transpose, "base": base}


def _write(name, new, kv, kv_heads, dim, cache, block=16, fused=False):
    return {"name": name, "kind": "write", "new": _text(new), "kv": _text(kv), "kv_heads": kv_heads, "dim": dim,
            "cache": cache, "block": block, "fused": fused}


def _read(name, new, kv, kv_heads, dim, cache, block=16, dtype="bf16"):
    """The last `new` of `kv` tokens of each sequence."""
    return {"name": name, "kind": "read", "new": _text(new), "kv": _text(kv), "kv_heads": kv_heads, "dim": dim,
            "cache": cache, "block": block, "dtype": dtype}


def _prompt(name, new, kv, heads, kv_heads, dim, cache, block=16):
    return {"name": name, "kind": "prompt", "new": _text(new), "kv": _text(kv), "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "cache": cache, "block": block}


def _decode(name, kv, heads, kv_heads, dim, cache, block=16, groups=(), prefix=()):
    """groups: sizes of the consecutive groups that share a prefix of `prefix` tokens."""
    return {"name": name, "kind": "decode", "kv": _text(kv), "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "cache": cache, "block": block, "groups": _text(groups), "prefix": _text(prefix)}


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _spread(seed, n, lo, hi):
    """n lengths between lo and hi, even over their logarithm."""
    r = random.Random(seed)
    return [_log_int(r, lo, hi) for _ in range(n)]


def listed():
    ages = _spread(5, 64, 1, 8000)
    return [
        # The new token of each of 64 requests, positions from the lengths on the device.
        _rope("rope_64tokens", [1] * 64, ages, 16, 4, 128, 128),
        # The longest prompt the model takes, beyond the length it was trained at, read in place from one projection.
        _rope("rope_32768_parts", [32768], [32768], 16, 4, 128, 128, scaling="parts,4,8192,1,32", fused=True, base=5e5),
        # A training step's gradient in fp32: neighbouring pairs, three quarters of the head, positions of packed documents.
        _rope("rope_grad_f32", [1791, 640, 257], [1791, 640, 257], 8, 8, 64, 48, "pairs", "f32", scattered=True,
              transpose=True),
        # The new token of each of 64 requests goes into its block, among tokens that are there.
        _write("write_64tokens_int8", [1] * 64, ages, 8, 128, "int8"),
        # The suffixes of the mixed batch, slices of one projection.
        _write("write_varlen16_e4m3", VARLEN_NEW, VARLEN_N, 8, 128, "e4m3", fused=True),
        # A long prompt into large blocks.
        _write("write_32768_int8_b64", [32768], [32768], 4, 128, "int8", 64),
        # A resumed request's cached prefix goes to a layer that wants it packed.
        _read("read_3328_e4m3", [3328], [3328], 2, 128, "e4m3"),
        # The mixed batch's whole caches come back in 16 bits.
        _read("read_varlen16_int8", VARLEN_N, VARLEN_N, 8, 128, "int8"),
        # A reloaded prompt's strict-prefix suffix: few rows, where latency counts.
        _prompt("resume_256_at_3328_int8", [256], [3584], 8, 2, 128, "int8"),
        # A mixed batch: cold prompts, full and partial prefix hits in one call.
        _prompt("resume_varlen16_e4m3", VARLEN_NEW, VARLEN_N, 8, 2, 128, "e4m3"),
        # One generated token of one request: the smallest attention call there is.
        _decode("decode_1seq_3584_e4m3", [3584], 8, 2, 128, "e4m3"),
        # Unrelated requests of every age, one of them at the longest context.
        _decode("decode_96seq_ragged_int8", [32768, 1] + _spread(4, 94, 17, 20000), 16, 4, 128, "int8"),
    ]


def _cut(rng, total, most, n):
    """n ragged lengths of about `total` tokens, each at most `most`."""
    w = [rng.random() + 0.02 for _ in range(n)]
    return [min(most, max(1, int(total * x / sum(w)))) for x in w]


def _draw_one(rng):
    kind = rng.choice(["rope", "rope", "write", "write", "read", "prompt", "prompt", "decode", "decode", "shared"])
    cache, block = rng.choice(["e4m3", "int8"]), rng.choice([16, 16, 16, 32, 64, 128, 256])
    kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 4), (8, 1), (3, 2), (2, 16), (5, 1), (4, 7)])
    dim, heads = rng.choice([64, 128, 128]), kv_heads * group
    if kind == "rope":
        d = rng.choice([64, 80, 128, 128, 256])
        rotary = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
        new = _cut(rng, _log_int(rng, 1, 16384), 16384, rng.randint(1, 32))
        scaling = rng.choice(["", "", "linear,4", "base,8", "parts,8,4096,1,32"])
        return _rope("", new, [n + _log_int(rng, 1, 100000) for n in new], heads, kv_heads, d, rotary,
                     rng.choice(["halves", "pairs"]), rng.choice(["bf16", "bf16", "f32"]), scaling, rng.random() < 0.4,
                     rng.random() < 0.4, rng.random() < 0.3, rng.choice([1e4, 5e5]))
    if kind in ("write", "read"):
        new = _cut(rng, _log_int(rng, 1, 40000), 16384, rng.randint(1, 64))
        kv = [n + rng.choice([0, rng.randint(0, 40), rng.randint(0, 2000)]) for n in new]
        if kind == "write":
            return _write("", new, kv, kv_heads, dim, cache, block, rng.random() < 0.5)
        return _read("", new, kv, kv_heads, dim, cache, block, rng.choice(["bf16", "bf16", "f32"]))
    if kind == "prompt":
        total = _log_int(rng, 16, 16384)
        new = _cut(rng, total, 12000, rng.randint(1, max(1, min(24, total // 24))))
        return _prompt("", new, [n + _log_int(rng, 1, 4096) for n in new], heads, kv_heads, dim, cache, block)
    if kind == "decode":
        n = _log_int(rng, 1, 128)
        return _decode("", [_log_int(rng, 1, 16000 if n < 48 else 6000) for _ in range(n)], heads, kv_heads, dim, cache,
                       block)
    groups = [_log_int(rng, 1, 64) for _ in range(rng.randint(1, 4))]
    prefix = [block * _log_int(rng, 1, 8192 // block) for _ in groups]
    kv = [p + _log_int(rng, 1, 1024) for g, p in zip(groups, prefix) for _ in range(g)]
    return _decode("", kv, heads, kv_heads, dim, cache, block, groups, prefix)


def draw(rng):
    costliest = max(work(c)["flops"] for c in listed())
    while True:
        c = _draw_one(rng)
        if work(c)["flops"] <= costliest:
            c.pop("name")
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (2 ** 31) + 41)
    return g


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[name]


def _size(name):
    return {"bf16": 2, "f32": 4}[name]


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device=DEV)


def _offsets(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def _up(a, b):
    return -(-a // b)


def _keys(gen, shape):
    """Keys with a few strong channels."""
    k = torch.randn(shape, generator=gen, device=DEV)
    return k * (1.0 + 4.0 * (torch.arange(shape[-1], device=DEV) % 16 == 3))


def _scale_of(most, cache):
    """The scale of values up to `most`, exact in 32 bits."""
    if cache == "e4m3":
        m, e = torch.frexp(most)
        e = torch.where(most > 0, torch.where(m <= 0.875, e - 9, e - 8), -127)
        s = ((e + 127) << 23).to(torch.int32).view(torch.float32)
    else:
        s = (most.double() / 127.0).float()
        s = ((s.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32)
    return s.clamp(min=LEAST)


def _codes(x, cache):
    """Codes of quotients, to nearest even."""
    x = x.clamp(-MOST[cache], MOST[cache])
    return x.float().to(torch.float8_e4m3fn) if cache == "e4m3" else x.round().to(torch.int8)


def _part_bytes(case):
    return case["kv_heads"] * case["block"] * case["dim"]


def _scales_at(case):
    """Offset of the used layer's key scales in a block; its value scales follow."""
    return 2 * LAYERS * _part_bytes(case) + 2 * 4 * case["kv_heads"]


def _part(case, cache, half):
    """The used layer's key (0) or value (1) codes: [blocks, kv heads, block tokens, dim]."""
    at = (2 + half) * _part_bytes(case)
    x = cache[:, at:at + _part_bytes(case)].view(_type(case["cache"]))
    return x.unflatten(1, (case["kv_heads"], case["block"], case["dim"]))


def _scales(case, cache, half):
    """And its scales: fp32 [blocks, kv heads]."""
    at = _scales_at(case) + half * 4 * case["kv_heads"]
    return cache[:, at:at + 4 * case["kv_heads"]].view(torch.float32)


def _cache(case, gen, blocks):
    """A cache of bytes [blocks, block_bytes], the used layer filled."""
    H, bt, d = case["kv_heads"], case["block"], case["dim"]
    size = _up(2 * LAYERS * _part_bytes(case) + 2 * LAYERS * 4 * H, 16) * 16
    cache = torch.zeros((blocks, size), dtype=torch.uint8, device=DEV)
    for half in (0, 1):
        for a in range(0, blocks, 4096):                      # in pieces: the values are fp32
            n = min(4096, blocks - a)
            x = _keys(gen, (n, H, bt, d)) if half == 0 else torch.randn((n, H, bt, d), generator=gen, device=DEV)
            x *= torch.rand((n, H, 1, 1), generator=gen, device=DEV) + 0.5
            s = _scale_of(x.abs().amax((2, 3)), case["cache"])
            _scales(case, cache, half)[a:a + n] = s
            to, code = _part(case, cache, half)[a:a + n], _codes(x / s[:, :, None, None], case["cache"])
            to.view(torch.int8).copy_(code.view(torch.int8))
    return cache


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
    kind, d, H = case["kind"], case["dim"], case["kv_heads"]
    kv = _ints(case["kv"])
    new = _ints(case["new"]) if "new" in case else [1] * len(kv)
    T = sum(new)
    s = {"case": case, "kv": kv, "kv_dev": _i32(kv), "new": new, "cu": _i32(_offsets(new))}
    if kind in ("rope", "write"):
        td = _type(case.get("dtype", "bf16"))
        Hq = case["heads"] if kind == "rope" else H
        # queries and keys, or keys and values, with what the projection has behind them
        x = torch.randn((T, Hq + 2 * H, d), generator=gen, device=DEV)
        at = Hq if kind == "rope" else 0
        x[:, at:at + H] = _keys(gen, (T, H, d))
        if kind == "write":
            x *= torch.rand((T, 1, 1), generator=gen, device=DEV) + 0.5
        x = x.to(td)
        a, b = x[:, :Hq], x[:, Hq:Hq + H]
        s["a"], s["b"] = (a, b) if case["fused"] else (a.contiguous(), b.contiguous())
        if kind == "rope":
            s["ya"], s["yb"] = torch.empty_like(s["a"].contiguous()), torch.empty_like(s["b"].contiguous())
            if case["scattered"]:
                s["pos"] = torch.randint(0, max(kv), (T,), generator=gen, device=DEV, dtype=torch.int32)
            return s
    if kind == "decode":
        groups, prefix = _ints(case["groups"]), _ints(case["prefix"])
        shared = list(zip(_offsets(groups), groups, prefix))
        s["cu_group"], s["prefix"] = _i32(_offsets(groups)), _i32(prefix)
    s["table"], blocks = _tables(case, kv, gen, shared if kind == "decode" else ())
    s["cache"] = _cache(case, gen, blocks)
    if kind in ("prompt", "decode"):
        s["q"] = torch.randn((T, case["heads"], d), generator=gen, device=DEV).to(torch.bfloat16)
    if kind == "read":
        s["ya"], s["yb"] = (torch.empty((T, H, d), dtype=_type(case["dtype"]), device=DEV) for _ in (0, 1))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2609_15030_amd import api
    from paper_2609_15030_amd import linattn as la
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rope":
        if "rope" not in s:      # frequencies on the device: what a program keeps
            words = c["scaling"].split(",")
            scaling = la.make_rope_scaling(words[0], *map(float, words[1:])) if c["scaling"] else None
            s["rope"] = api.Rope(c["dim"], c["rotary"], c["layout"], c["base"], scaling)
        where = {"positions": s["pos"]} if c["scattered"] else {"cu_seqlens": s["cu"], "kv_len": s["kv_dev"]}
        s["rope"].apply(s["a"], s["b"], s["ya"], s["yb"], transpose=c["transpose"], **where)
        return [s["ya"], s["yb"]]
    if "layer" not in s:
        part, scales = _part_bytes(c), _scales_at(c)
        s["layer"] = la.make_kv_layer(s["cache"], s["table"], c["block"], c["kv_heads"], c["dim"], _type(c["cache"]),
                                      k_offset=2 * part, v_offset=3 * part, k_scales=scales,
                                      v_scales=scales + 4 * c["kv_heads"])
    if kind == "write":
        la.la_kv_write(s["layer"], s["a"], s["b"], s["cu"], s["kv_dev"])
        return _written(s)
    if kind == "read":
        la.la_kv_read(s["layer"], s["ya"], s["yb"], s["cu"], s["kv_dev"])
        return [s["ya"], s["yb"]]
    if kind == "prompt":
        if "plan" not in s:      # lengths, workspace
            s["plan"] = api.AttnPrefill(c["heads"], c["kv_heads"], c["dim"], s["new"], s["kv"])
        return [s["plan"].run_paged(s["layer"], s["q"])]
    if "plan" not in s:
        s["plan"] = api.AttnDecode(len(s["kv"]), c["heads"], c["kv_heads"], c["dim"], max(s["kv"]),
                                   cu_group=s["cu_group"] if c["groups"] else None,
                                   max_prefix_len=max(_ints(c["prefix"]) or [0]))
    return [s["plan"].run(s["layer"], s["q"], s["kv_dev"], s["prefix"] if c["groups"] else None)]


def _written(s):
    """Codes and scales: a code is a whole number of scales (int8), or the value it stands for by itself (e4m3)."""
    return [f(s["case"], s["cache"], half) for half in (0, 1) for f in (_part, _scales)]


def _places(s):
    """Sequence and position of each new token."""
    cu = s["cu"].long()
    n = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEV), n, output_size=sum(s["new"]))
    return seq, torch.arange(sum(s["new"]), device=DEV) - cu[seq] + (s["kv_dev"].long() - n)[seq]


def _frequencies(case):
    """Radians a token, of each pair, in 64 bits."""
    r = case["rotary"]
    i = torch.arange(r // 2, device=DEV, dtype=torch.float64)
    words = case["scaling"].split(",")
    kind, num = words[0], [float(w) for w in words[1:]]
    base = case["base"] * (num[0] ** (r / (r - 2)) if kind == "base" and r > 2 else 1.0)
    f = base ** (-2.0 * i / r)
    if kind == "linear":
        f = f / num[0]
    if kind == "parts":
        keep = ((num[1] * f / (2 * math.pi) - num[2]) / (num[3] - num[2])).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / num[0])
    return f


def _rotate(x, cos, sin, r, layout):
    y = x.float()
    if layout == "halves":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos, y[..., r:]], -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        y = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), y[..., r:]], -1)
    return y.to(x.dtype)


def _pad(x, cu, most):
    """Packed rows as [sequences, most, ...], zeros behind each sequence's end."""
    at = torch.arange(most, device=DEV)[None, :]
    n = (cu[1:] - cu[:-1])[:, None]
    rows = (cu[:-1, None] + at).clamp(max=x.shape[0] - 1)
    return x.float()[rows.long()] * (at < n).reshape(n.shape[0], most, *[1] * (x.dim() - 1))


def _gather(s, half, most):
    """Keys or values of every sequence: [sequences, most, kv heads, dim] in 32 bits."""
    c = s["case"]
    ids = s["table"].long().clamp(min=0)
    x = _part(c, s["cache"], half)[ids].float() * _scales(c, s["cache"], half)[ids][..., None, None]
    return x.transpose(2, 3).flatten(1, 2)[:, :most]


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
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rope":
        pos = s["pos"] if c["scattered"] else _places(s)[1]
        angle = pos.double()[:, None] * _frequencies(c)
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        sin = -sin if c["transpose"] else sin
        return [_rotate(s[x], cos, sin, c["rotary"], c["layout"]) for x in ("a", "b")]
    if kind == "write":
        return _plain_write(s)
    most, kv_len, scale = max(s["kv"]), s["kv_dev"], c["dim"] ** -0.5
    if kind == "read":
        seq, pos = _places(s)
        block, slot = s["table"][seq, pos // c["block"]].long(), pos % c["block"]
        return [(_part(c, s["cache"], h)[block, :, slot].float() * _scales(c, s["cache"], h)[block][..., None])
                .to(_type(c["dtype"])) for h in (0, 1)]
    if kind == "decode":
        o = _attend(s["q"].float()[:, None], _gather(s, 0, most), _gather(s, 1, most), kv_len[:, None] - 1, kv_len, scale)
        return [o[:, 0].to(torch.bfloat16)]
    rows, cu = max(s["new"]), s["cu"]
    n = (cu[1:] - cu[:-1])[:, None]
    pos = torch.arange(rows, device=DEV)[None, :] + (kv_len[:, None] - n)
    o = _attend(_pad(s["q"], cu, rows), _gather(s, 0, most), _gather(s, 1, most), pos, kv_len, scale)
    seq, at = _places(s)
    return [o[seq, at - (kv_len - n[:, 0])[seq]].to(torch.bfloat16)]


def _plain_write(s):
    c = s["case"]
    H, bt, d = c["kv_heads"], c["block"], c["dim"]
    seq, pos = _places(s)
    slot = pos % bt
    ids, at = torch.unique(s["table"][seq, pos // bt].long(), return_inverse=True)      # blocks, each token's block
    first = torch.full((len(ids),), bt, device=DEV).scatter_reduce(0, at, slot, "amin")
    stays = torch.arange(bt, device=DEV) < first[:, None]                               # tokens that stay
    for half, x in ((0, s["a"]), (1, s["b"])):
        x = x.float()
        most = torch.zeros((len(ids), H), device=DEV).scatter_reduce(0, at[:, None].expand(-1, H), x.abs().amax(-1), "amax")
        codes, scales = _part(c, s["cache"], half), _scales(c, s["cache"], half)
        old, new = scales[ids], _scale_of(most, c["cache"])
        new = torch.where(first[:, None] > 0, torch.maximum(old, new), new)
        there = codes.view(torch.int8)[ids]
        # quotients in 64 bits: ties to even have to be seen as ties
        moved = there.view(codes.dtype).double() * (old.double() / new.double())[..., None, None]
        if c["cache"] == "int8":
            moved = there.view(codes.dtype).double() * old.double()[..., None, None] / new.double()[..., None, None]
        moved = torch.where(stays[:, None, :, None], _codes(moved, c["cache"]).view(torch.int8), there)
        codes.view(torch.int8)[ids] = moved
        codes.view(torch.int8)[ids[at], :, slot] = _codes(x.double() / new.double()[at][..., None], c["cache"]).view(torch.int8)
        scales[ids] = new
    return _written(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    d, H, kv, kind = case["dim"], case["kv_heads"], _ints(case["kv"]), case["kind"]
    new = _ints(case["new"]) if "new" in case else [1] * len(kv)
    if kind == "rope":
        values = sum(new) * (case["heads"] + H) * d
        return {"bytes": 2.0 * values * _size(case["dtype"]), "flops": 3.0 * values * case["rotary"] / d}
    blocks = sum(_up(n, case["block"]) for n in kv)
    touched = sum(_up(n, case["block"]) - (n - m) // case["block"] for n, m in zip(kv, new))
    if kind == "write":
        return {"bytes": 2.0 * sum(new) * H * d * 3 + 8.0 * H * touched, "flops": 4.0 * sum(new) * H * d}
    if kind == "read":
        return {"bytes": 2.0 * sum(new) * H * d * (1 + _size(case["dtype"])) + 8.0 * H * touched,
                "flops": 2.0 * sum(new) * H * d}
    heads = case["heads"]
    if kind == "decode":
        groups, prefix = _ints(case["groups"]), _ints(case["prefix"])
        again = sum((g - 1) * p for g, p in zip(groups, prefix))       # read once for its group
        return {"bytes": 2.0 * (sum(kv) - again) * H * d + 8.0 * H * (blocks - again // case["block"])
                + 4.0 * len(kv) * heads * d, "flops": 4.0 * d * heads * sum(kv)}
    pairs = sum(n * (L - n) + n * (n + 1) / 2 for n, L in zip(new, kv))
    return {"bytes": 4.0 * sum(new) * heads * d + 2.0 * sum(kv) * H * d + 8.0 * H * blocks,
            "flops": 4.0 * d * heads * pairs}


# ---------------------------------------------------------------------------
# 64-bit results, from the definition
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


def _exact_rope(s):
    """Pairs as complex numbers, turned."""
    c = s["case"]
    r = c["rotary"]
    pos = []
    for n, L in zip(s["new"], s["kv"]):
        pos += range(L - n, L)
    pos = s["pos"].double() if c["scattered"] else torch.tensor(pos, dtype=torch.float64, device=DEV)
    angle = torch.outer(pos, _frequencies(c)) * (-1.0 if c["transpose"] else 1.0)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    outs = []
    for x in (s["a"].double(), s["b"].double()):
        pairs = x[..., :r].unflatten(-1, (2, r // 2) if c["layout"] == "halves" else (r // 2, 2))
        pairs = pairs.transpose(-1, -2) if c["layout"] == "halves" else pairs
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.transpose(-1, -2) if c["layout"] == "halves" else z
        outs.append(torch.cat([z.flatten(-2), x[..., r:]], -1))
    return outs


def _exact_scale(most, cache):
    """The scale of a block's values, in 64 bits: a power of two, or one of 8 significant bits, not below most / the largest code."""
    x = most / MOST[cache]
    e = torch.floor(torch.log2(x.clamp(min=LEAST)))
    if cache == "int8":
        step = _two_to(e - 7)
        return (torch.ceil(x / step) * step).clamp(min=LEAST)
    return torch.where(_two_to(e) < x, _two_to(e + 1), _two_to(e)).clamp(min=LEAST)


def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_write(s):
    c = s["case"]
    bt, cache = c["block"], c["cache"]
    table = s["table"].cpu().tolist()
    outs = []
    for half, x in ((0, s["a"].double()), (1, s["b"].double())):
        codes = _part(c, s["cache"], half).double()
        scales = _scales(c, s["cache"], half).double()
        row = 0
        for i, (n, L) in enumerate(zip(s["new"], s["kv"])):
            p = L - n
            while p < L:
                end = min(L, (p // bt + 1) * bt)
                b, a = table[i][p // bt], p % bt
                y = x[row:row + end - p].transpose(0, 1)                                  # [heads, tokens, dim]
                scale = _exact_scale(y.abs().amax((1, 2)), cache)
                if a:
                    scale = torch.maximum(scale, scales[b])
                    codes[b, :, :a] = _exact_codes(codes[b, :, :a] * scales[b][:, None, None] / scale[:, None, None], cache)
                codes[b, :, a:a + end - p] = _exact_codes(y / scale[:, None, None], cache)
                scales[b] = scale
                row, p = row + end - p, end
        outs += [codes, scales]
    return outs


def _exact_codes(x, cache):
    if cache == "int8":
        return torch.round(x)
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))      # steps of 2^-3 in each power of two, of 2^-9 below 2^-6
    return torch.round(x * _two_to(3 - e)) * _two_to(e - 3)


def exact(case, seed):
    s = prepare(case, seed)
    kind, kv, new = case["kind"], s["kv"], s["new"]
    if kind == "rope":
        return _exact_rope(s)
    if kind == "write":
        return _exact_write(s)
    outs, at = None, 0
    for i, (n, L) in enumerate(zip(new, kv)):
        ids = s["table"][i, :_up(L, case["block"])].long()
        k, v = ((_part(case, s["cache"], h)[ids].double() * _scales(case, s["cache"], h)[ids].double()[:, :, None, None])
                .transpose(1, 2).flatten(0, 1)[:L] for h in (0, 1))
        if kind == "read":
            outs = [[], []] if outs is None else outs
            outs[0].append(k[L - n:])
            outs[1].append(v[L - n:])
            continue
        if outs is None:
            outs = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        G = case["heads"] // case["kv_heads"]
        for h in range(case["heads"]):
            outs[at:at + n, h] = _exact_rows(s["q"][at:at + n, h].double(), k[:, h // G].contiguous(),
                                             v[:, h // G].contiguous(), L - n)
        at += n
    return [torch.cat(x) for x in outs] if kind == "read" else [outs]
