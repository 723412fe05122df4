"""Attention over packed and cached keys, and writes into the cache, against the
fp64 oracle (oracle/attention.py), with the bound that its docstring derives.

Sizes sit around the kernels' edges: tiles of 16, 64 and 256 rows, key tiles of
16, 32 and 64, parts of 512 keys, blocks of 16 to 256 tokens, one to many heads
per key head, sequences of no token, tokens without a key."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen)


def _host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _check(o, parts, d, bf16, what):
    """parts: (first row, (o, mean, size), keys) of every sequence."""
    got, worst = _host(o), 0.0
    for at, (ref, mean, size), keys in parts:
        n = ref.shape[0]
        tol = oa.tolerance(ref, mean, size, keys, d, bf16)
        diff = np.abs(got[at:at + n] - ref)
        assert np.all(np.isfinite(got[at:at + n])), what
        worst = max(worst, float(np.max(diff / tol, initial=0.0)))
    print(f"[attn] {what}: worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, (what, worst)


class Cache:
    """Keys and values of `kv` tokens a sequence in blocks of a shared cache."""

    def __init__(self, gen, kv, heads, d, kind, bt, layers=3, layer=1, spare=3, shared=()):
        self.kv, self.heads, self.d, self.kind, self.bt = kv, heads, d, kind, bt
        self.scales = (0.37, 0.11) if kind == "fp8" else (1.0, 1.0)
        need = [-(-n // bt) for n in kv]
        blocks = sum(need) + spare
        perm = torch.randperm(blocks, generator=gen).to(torch.int32)
        self.table = torch.full((len(kv), max(need + [1])), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = perm[at:at + n]
            at += n
        for first, n, tokens in shared:            # rows first + 1 .. first + n - 1 begin with row first's blocks
            self.table[first:first + n, :-(-tokens // bt)] = self.table[first, :-(-tokens // bt)].clone()
        size = torch.empty(0, dtype=TYPES[kind]).element_size()
        self.part_bytes = heads * bt * d * size
        self.off = (2 * layer * self.part_bytes, (2 * layer + 1) * self.part_bytes)
        bytes_ = torch.zeros((blocks, 2 * layers * self.part_bytes), dtype=torch.uint8)
        for half in (0, 1):
            x = _rand(gen, blocks, heads, bt, d) / self.scales[half]
            self.part(bytes_, half).copy_(x.to(TYPES[kind]))
        self.host = bytes_
        self.dev = bytes_.cuda()
        self.table_dev = self.table.cuda()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def part(self, bytes_, half):
        o = self.off[half]
        return bytes_[:, o:o + self.part_bytes].view(TYPES[self.kind]).unflatten(1, (self.heads, self.bt, self.d))

    def layer(self):
        return la.make_kv_layer(self.dev, self.table_dev, self.bt, self.heads, self.d, TYPES[self.kind], self.off[0],
                                self.off[1], self.scales[0], self.scales[1], self.err)

    def rows(self, seq):
        """(k, v) of a sequence in fp64, as the stored values stand for (scales as the fp32 the call takes)."""
        return tuple(oa.table_rows(_host(self.part(self.host, h)), self.table.numpy(), seq, self.kv[seq], self.bt,
                                   float(np.float32(self.scales[h]))) for h in (0, 1))


# --- prompts over packed keys --------------------------------------------------

PROMPTS = [
    # new tokens, q heads, kv heads, d, type, sliced
    ([1], 1, 1, 64, "bf16", False),
    ([5, 0, 1, 64], 4, 2, 128, "bf16", False),
    ([63, 65, 17], 8, 8, 128, "bf16", True),
    ([300], 6, 2, 64, "bf16", False),
    ([129, 2, 257], 16, 1, 128, "bf16", True),
    ([520], 2, 1, 128, "bf16", False),
    ([1], 1, 1, 128, "f32", False),
    ([33, 0, 31, 100], 6, 3, 64, "f32", True),
    ([70, 129], 4, 1, 128, "f32", False),
]


def _packed(case, seed, q=None):
    new, hq, hk, d, kind, sliced = case
    gen = torch.Generator().manual_seed(seed)
    T = sum(new)
    x = _rand(gen, T, hq + 2 * hk + (2 if sliced else 0), d).to(TYPES[kind]).cuda()
    parts = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:hq + 2 * hk]
    return parts if sliced else tuple(p.contiguous() for p in parts)


def _packed_ref(case, q, k, v, scale):
    out, at = [], 0
    for n in case[0]:
        out.append((at, oa.attend(_host(q[at:at + n]), _host(k[at:at + n]), _host(v[at:at + n]), 0, scale), max(n, 1)))
        at += n
    return out


@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: f"{c[0]}-{c[1]}/{c[2]}x{c[3]}-{c[4]}{'-sliced' if c[5] else ''}")
def test_prompts(case):
    new, hq, hk, d, kind, _ = case
    q, k, v = _packed(case, 11)
    o = api.AttnPrefill(hq, hk, d, new, dtype=TYPES[kind]).run(q, k, v)
    torch.cuda.synchronize()
    _check(o, _packed_ref(case, q, k, v, float(np.float32(d ** -0.5))), d, kind == "bf16", str(case))


def test_prompt_of_large_scores():
    """Scores far apart: the running maximum moves by hundreds between tiles."""
    case = ([400], 4, 2, 128, "bf16", False)
    q, k, v = _packed(case, 12)
    ramp = torch.linspace(0.1, 30.0, 400, device="cuda").to(torch.bfloat16)
    k = k * ramp[:, None, None]
    o = api.AttnPrefill(4, 2, 128, [400], scale=0.7).run(q, k, v)
    torch.cuda.synchronize()
    _check(o, _packed_ref(case, q, k, v, float(np.float32(0.7))), 128, True, "large scores")


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_unseen_infinities_and_nan_have_no_effect(kind, d):
    """Keys and values of later tokens, made infinite or NaN, leave the earlier
    rows' bits alone; the rows that see them show it."""
    case = ([333], 4, 2, d, kind, False)
    q, k, v = _packed(case, 13)
    plan = api.AttnPrefill(4, 2, d, [333], dtype=TYPES[kind])
    clean = plan.run(q, k, v).clone()
    k2, v2 = k.clone(), v.clone()
    k2[200] = float("nan")
    v2[200, :, 3] = float("inf")
    v2[270, :, 7] = float("nan")
    v2[290, :, 9] = -float("inf")
    k2[300] = float("inf")
    v2[320] = float("nan")
    o = plan.run(q, k2, v2)
    torch.cuda.synchronize()
    assert torch.equal(o[:200], clean[:200])
    assert torch.isnan(o[200:]).all()
    # values only: the columns that are finite stay, the others take the value
    v3 = v.clone()
    v3[201, :, 3] = float("inf")
    v3[202, :, 5] = float("nan")
    o = plan.run(q, k, v3)
    torch.cuda.synchronize()
    other = [c for c in range(d) if c not in (3, 5)]
    assert torch.equal(o[:, :, other], clean[:, :, other])
    assert torch.equal(o[:201], clean[:201])
    assert torch.isposinf(o[201:, :, 3]).all() and torch.isnan(o[202:, :, 5]).all()
    assert torch.equal(o[201, :, 5], clean[201, :, 5])


# --- prompts over cached keys --------------------------------------------------

RESUMES = [
    # new tokens, keys, q heads, kv heads, d, io, cache, block tokens
    ([1], [1], 1, 1, 64, "bf16", "bf16", 16),
    ([1, 16, 0], [40, 16, 7], 4, 2, 128, "bf16", "bf16", 16),
    ([70, 5], [700, 513], 8, 2, 128, "bf16", "bf16", 32),
    ([256], [600], 8, 2, 128, "bf16", "fp8", 16),
    ([65, 3, 130], [65, 1000, 257], 6, 3, 64, "bf16", "fp8", 64),
    ([33, 40], [33, 290], 16, 1, 64, "bf16", "bf16", 256),
    ([20, 33], [90, 300], 4, 2, 128, "f32", "f32", 16),
    ([64], [129], 3, 3, 64, "f32", "f32", 128),
    ([12, 30], [5, 0], 4, 2, 128, "bf16", "bf16", 16),        # more tokens than keys: the first see none
]


def _resume(case, seed):
    new, kv, hq, hk, d, io, kind, bt = case
    gen = torch.Generator().manual_seed(seed)
    return _rand(gen, sum(new), hq, d).to(TYPES[io]).cuda(), Cache(gen, kv, hk, d, kind, bt)


def _resume_ref(case, q, cache, scale):
    out, at = [], 0
    for i, (n, L) in enumerate(zip(case[0], case[1])):
        k, v = cache.rows(i)
        out.append((at, oa.attend(_host(q[at:at + n]), k, v, L - n, scale), max(L, 1)))
        at += n
    return out


@pytest.mark.parametrize("case", RESUMES, ids=lambda c: f"{c[0]}of{c[1]}-{c[2]}/{c[3]}x{c[4]}-{c[6]}-b{c[7]}")
def test_resumed_prompts(case):
    new, kv, hq, hk, d, io, kind, bt = case
    q, cache = _resume(case, 21)
    o = api.AttnPrefill(hq, hk, d, new, kv, TYPES[io]).run_paged(cache.layer(), q)
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    _check(o, _resume_ref(case, q, cache, float(np.float32(d ** -0.5))), d, io == "bf16", str(case))


def test_cache_slots_behind_a_sequence_have_no_effect():
    """Stale bytes (here NaN) in the slots past each sequence's last key."""
    case = ([30, 70], [133, 290], 4, 2, 128, "bf16", "bf16", 64)
    q, cache = _resume(case, 22)
    plan = api.AttnPrefill(4, 2, 128, case[0], case[1])
    dec = api.AttnDecode(2, 4, 2, 128, 290)
    kv = torch.tensor(case[1], dtype=torch.int32, device="cuda")
    a, b = plan.run_paged(cache.layer(), q).clone(), dec.run(cache.layer(), q[:2].contiguous(), kv).clone()
    for i, n in enumerate(case[1]):
        last = int(cache.table[i, (n - 1) // 64])
        for half in (0, 1):
            cache.part(cache.dev, half)[last, :, n % 64:] = float("nan")
    assert torch.equal(plan.run_paged(cache.layer(), q), a)
    assert torch.equal(dec.run(cache.layer(), q[:2].contiguous(), kv), b)


# --- single tokens -------------------------------------------------------------

DECODES = [
    # keys, q heads, kv heads, d, io, cache, block tokens, group sizes, prefixes
    ([1], 1, 1, 64, "bf16", "bf16", 16, (), ()),
    ([0, 1, 15, 16, 17, 31, 33], 8, 2, 128, "bf16", "bf16", 16, (), ()),
    ([511, 512, 513, 1025, 3], 4, 4, 128, "bf16", "bf16", 32, (), ()),
    ([700, 40, 1300], 16, 1, 128, "bf16", "fp8", 16, (), ()),
    ([300, 20], 40, 2, 64, "bf16", "fp8", 64, (), ()),
    ([260, 1, 600], 6, 3, 128, "f32", "f32", 16, (), ()),
    ([33, 530], 4, 1, 64, "f32", "f32", 256, (), ()),
    ([100, 97, 130, 128], 4, 2, 128, "bf16", "bf16", 16, (4,), (96,)),
    ([1200, 1100, 1030, 50, 60, 9], 8, 2, 128, "bf16", "bf16", 32, (3, 2), (1024, 32)),
    ([700, 610, 600, 640, 20], 16, 2, 64, "bf16", "fp8", 16, (1, 3), (640, 593)),  # a group of one, a prefix inside a block
    ([200, 90, 300, 150], 6, 3, 128, "f32", "f32", 16, (4,), (128,)),              # a member shorter than the prefix
    ([40] * 70, 2, 1, 64, "bf16", "bf16", 16, (70,), (32,)),                       # more rows than one tile
]


@pytest.mark.parametrize("case", DECODES, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}/{c[2]}x{c[3]}-{c[5]}-b{c[6]}-g{len(c[7])}")
def test_single_tokens(case):
    kv, hq, hk, d, io, kind, bt, groups, prefix = case
    gen = torch.Generator().manual_seed(31)
    q = _rand(gen, len(kv), hq, d).to(TYPES[io]).cuda()
    starts = np.concatenate([[0], np.cumsum(groups)]).astype(np.int32)
    cache = Cache(gen, kv, hk, d, kind, bt, shared=[(int(s), n, p) for s, n, p in zip(starts, groups, prefix)])
    kv_dev = torch.tensor(kv, dtype=torch.int32, device="cuda")
    cu = torch.from_numpy(starts).cuda() if groups else None
    pre = torch.tensor(prefix, dtype=torch.int32, device="cuda") if groups else None
    plan = api.AttnDecode(len(kv), hq, hk, d, max(kv), TYPES[io], cu_group=cu, max_prefix_len=max(prefix, default=0))
    o = plan.run(cache.layer(), q, kv_dev, pre).clone()
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    ref = []
    for i, n in enumerate(kv):
        k, v = cache.rows(i)
        ref.append((i, oa.attend(_host(q[i:i + 1]), k, v, n - 1, float(np.float32(d ** -0.5))), max(n, 1)))
    _check(o, ref, d, io == "bf16", str(case))
    # the same bits with spare room in the plan, and again
    wide = api.AttnDecode(len(kv), hq, hk, d, cache.table.shape[1] * bt, TYPES[io], cu_group=cu,
                          max_prefix_len=max(prefix, default=0))
    assert torch.equal(wide.run(cache.layer(), q, kv_dev, pre), o)
    assert torch.equal(plan.run(cache.layer(), q, kv_dev, pre), o)


def test_a_group_larger_than_its_plan():
    """The sequences behind max_group read their whole keys themselves."""
    gen = torch.Generator().manual_seed(33)
    kv = [300 + 7 * i for i in range(9)]
    cache = Cache(gen, kv, 2, 128, "bf16", 16, shared=[(0, 9, 288)])
    q = _rand(gen, 9, 16, 128).to(torch.bfloat16).cuda()
    kv_dev = torch.tensor(kv, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    pre = torch.tensor([288], dtype=torch.int32, device="cuda")
    for most in (1, 4):
        plan = api.AttnDecode(9, 16, 2, 128, max(kv), cu_group=cu, max_prefix_len=288, max_group=most)
        plan.workspace.fill_(0xFF)               # a slot that nothing wrote is NaN
        o = plan.run(cache.layer(), q, kv_dev, pre)
        ref = [(i, oa.attend(_host(q[i:i + 1]), *cache.rows(i), n - 1, float(np.float32(128 ** -0.5))), n) for i, n in enumerate(kv)]
        _check(o, ref, 128, True, f"max_group {most}")


# --- what a call may not depend on ---------------------------------------------

def test_a_single_token_does_not_depend_on_its_batch():
    gen = torch.Generator().manual_seed(41)
    kv = [700, 600, 33]
    cache = Cache(gen, kv, 2, 128, "bf16", 16)
    q = _rand(gen, 3, 8, 128).to(torch.bfloat16).cuda()
    kv_dev = torch.tensor(kv, dtype=torch.int32, device="cuda")
    batch = api.AttnDecode(3, 8, 2, 128, 700).run(cache.layer(), q, kv_dev).clone()
    for i in range(3):
        one = la.make_kv_layer(cache.dev, cache.table_dev[i:i + 1], 16, 2, 128, torch.bfloat16, *cache.off)
        assert torch.equal(api.AttnDecode(1, 8, 2, 128, 700).run(one, q[i:i + 1], kv_dev[i:i + 1].clone()), batch[i:i + 1])


@pytest.mark.parametrize("io,kind", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
def test_a_batch_of_every_length(io, kind):
    """70 sequences (more than one step of the item search), from none to many parts: a
    small call that splits its keys and a large one that takes sequences longest first
    give what the oracle does; each twice the same bits."""
    rng = np.random.default_rng(46)
    for n_seqs, rows, most in ((70, 3, 900), (12, 400, 2000)):
        new = [int(x) for x in rng.integers(0, rows + 1, n_seqs)]
        kv = [n + int(x) for n, x in zip(new, rng.integers(0, most, n_seqs))]
        case = (new, kv, 4, 2, 64, io, kind, 16)
        q, cache = _resume(case, 47)
        plan = api.AttnPrefill(4, 2, 64, new, kv, TYPES[io])
        o = plan.run_paged(cache.layer(), q).clone()
        torch.cuda.synchronize()
        assert torch.equal(plan.run_paged(cache.layer(), q), o)
        some = range(n_seqs) if rows < 10 else (0, 3, 7, 11)         # the oracle is slow: a few of the long ones
        ref, at = [], 0
        for i, (n, L) in enumerate(zip(new, kv)):
            if i in some:
                k, v = cache.rows(i)
                ref.append((at, oa.attend(_host(q[at:at + n]), k, v, L - n, 0.125), max(L, 1)))
            at += n
        _check(o, ref, 64, io == "bf16", f"{n_seqs} sequences, {kind}")


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_infinities_beside_the_end_of_a_prefix(io):
    """A prefix of 37 keys ends inside a run of 16: its last values and the first own
    ones, infinite or NaN, reach the column they stand in and no other."""
    gen = torch.Generator().manual_seed(48)
    kv = [90, 61, 37]
    cache = Cache(gen, kv, 2, 64, io, 16, shared=[(0, 3, 37)])
    q = _rand(gen, 3, 4, 64).to(TYPES[io]).cuda()
    kv_dev, cu, pre = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (kv, [0, 3], [37]))
    plan = api.AttnDecode(3, 4, 2, 64, 90, TYPES[io], cu_group=cu, max_prefix_len=37)
    clean = plan.run(cache.layer(), q, kv_dev, pre).clone()
    v = cache.part(cache.dev, 1)
    at = int(cache.table[0, 2])
    v[at, :, 34 - 32, 3] = float("inf")
    v[at, :, 36 - 32, 5] = float("nan")
    v[at, :, 37 - 32, 7] = -float("inf")             # the first own key of two of them; none of the third
    o = plan.run(cache.layer(), q, kv_dev, pre)
    torch.cuda.synchronize()
    assert torch.isposinf(o[:, :, 3]).all() and torch.isnan(o[:, :, 5]).all()
    assert torch.isneginf(o[:2, :, 7]).all() and torch.equal(o[2, :, 7], clean[2, :, 7])
    rest = [i for i in range(64) if i not in (3, 5, 7)]
    assert torch.equal(o[:, :, rest], clean[:, :, rest])


def test_missing_blocks_are_counted_and_read_as_zero():
    case = ([40], [200], 4, 2, 128, "bf16", "bf16", 16)
    q, cache = _resume(case, 42)
    cache.table[0, 3], cache.table[0, 7] = -1, cache.host.shape[0]
    cache.table_dev.copy_(cache.table)
    o = api.AttnPrefill(4, 2, 128, [40], [200]).run_paged(cache.layer(), q).clone()
    torch.cuda.synchronize()
    assert int(cache.err) >= 2
    _check(o, _resume_ref(case, q, cache, float(np.float32(128 ** -0.5))), 128, True, "missing blocks, prompt")
    cache.err.zero_()
    kv = torch.tensor([200], dtype=torch.int32, device="cuda")
    d = api.AttnDecode(1, 4, 2, 128, 200).run(cache.layer(), q[39:], kv)
    torch.cuda.synchronize()
    assert int(cache.err) >= 2
    _check(d, [(0, oa.attend(_host(q[39:]), *cache.rows(0), 199, float(np.float32(128 ** -0.5))), 200)], 128, True,
           "missing blocks, single token")
    # a kv_len past the plan's longest is cut there and counted
    cache.err.zero_()
    short = api.AttnDecode(1, 4, 2, 128, 150)
    cut = short.run(cache.layer(), q[39:], kv).clone()
    torch.cuda.synchronize()
    assert int(cache.err) >= 1
    assert torch.equal(cut, short.run(cache.layer(), q[39:], torch.full_like(kv, 150)))


def test_a_cache_past_32_bit_offsets():
    """Blocks beyond 4 GB of cache, of 1 MB each; the bytes before them are never touched."""
    hk, d, bt, n = 1, 128, 16, 37
    blocks = 4200
    cache = torch.empty((blocks, 1 << 20), dtype=torch.uint8, device="cuda")
    ids = [4199, 4100, 4098]
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    layer = la.make_kv_layer(cache, table, bt, hk, d, torch.bfloat16, k_offset=1 << 19)
    gen = torch.Generator().manual_seed(43)
    k, v, q = (_rand(gen, n, 1 if i < 2 else 4, d).to(torch.bfloat16).cuda() for i in range(3))
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    kv = torch.tensor([n], dtype=torch.int32, device="cuda")
    la.la_kv_write(layer, k, v, cu, kv)
    want = api.AttnPrefill(4, 1, d, [n]).run(q, k, v)
    got = api.AttnPrefill(4, 1, d, [n], [n]).run_paged(layer, q)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    one = api.AttnDecode(1, 4, 1, d, n).run(layer, q[n - 1:], kv)
    torch.cuda.synchronize()
    _check(one, [(0, oa.attend(_host(q[n - 1:]), _host(k), _host(v), n - 1, float(np.float32(d ** -0.5))), n)], d, True,
           "past 4 GB")


def test_another_stream():
    case = ([200], [700], 8, 2, 128, "bf16", "bf16", 16)
    q, cache = _resume(case, 44)
    plan, dec = api.AttnPrefill(8, 2, 128, [200], [700]), api.AttnDecode(1, 8, 2, 128, 700)
    kv = torch.tensor([700], dtype=torch.int32, device="cuda")
    qd = q[199:].contiguous()
    a, b = plan.run_paged(cache.layer(), q).clone(), dec.run(cache.layer(), qd, kv).clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    plan.o.zero_()
    dec.o.zero_()
    s.wait_stream(torch.cuda.current_stream())
    plan.run_paged(cache.layer(), q, stream=s)
    with torch.cuda.stream(s):
        dec.run(cache.layer(), qd, kv)
    s.synchronize()
    assert torch.equal(plan.o, a) and torch.equal(dec.o, b)


def test_a_captured_decode_follows_its_lengths():
    """One graph of a write and a decode step, replayed as lengths, tables and inputs change."""
    gen = torch.Generator().manual_seed(45)
    kv0, hq, hk, d, bt = [600, 33, 90], 8, 2, 128, 16
    cache = Cache(gen, [n + 8 for n in kv0], hk, d, "bf16", bt)
    kv = torch.tensor(kv0, dtype=torch.int32, device="cuda")
    cu = torch.arange(4, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((3, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk))
    plan, layer = api.AttnDecode(3, hq, hk, d, 608), cache.layer()
    la.la_kv_write(layer, k, v, cu, kv)
    plan.run(layer, q, kv)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        la.la_kv_write(layer, k, v, cu, kv)
        plan.run(layer, q, kv)
    for step in range(4):
        kv += 1
        for t in (q, k, v):
            t.copy_(_rand(gen, *t.shape).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = plan.o.clone()
        eager = api.AttnDecode(3, hq, hk, d, 608).run(layer, q, kv)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), step
    assert int(cache.err) == 0


# --- writes --------------------------------------------------------------------

@pytest.mark.parametrize("new,kv,hk,d,io,kind,bt,sliced", [
    ([1] * 70, list(range(1, 71)), 2, 128, "bf16", "bf16", 16, False),
    ([40, 0, 3, 129], [40, 9, 200, 300], 8, 128, "bf16", "bf16", 32, True),
    ([7, 100], [50, 100], 3, 64, "bf16", "fp8", 16, True),
    ([33, 1], [64, 17], 1, 64, "f32", "f32", 64, False),
    ([260], [700], 5, 128, "f32", "f32", 256, True),
])
def test_cache_writes(new, kv, hk, d, io, kind, bt, sliced):
    gen = torch.Generator().manual_seed(51)
    cache = Cache(gen, kv, hk, d, kind, bt)
    x = _rand(gen, sum(new), 2 * hk + (1 if sliced else 0), d).to(TYPES[io]).cuda()
    k, v = x[:, :hk], x[:, hk:2 * hk]
    if not sliced:
        k, v = k.contiguous(), v.contiguous()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    want = cache.host.clone()
    for half, src in ((0, k), (1, v)):
        y = src.float().cpu() / torch.tensor(cache.scales[half])
        y = y.clamp(-448, 448).to(TYPES[kind])
        to, at = cache.part(want, half), 0
        for i, (n, L) in enumerate(zip(new, kv)):
            for t in range(n):
                pos = L - n + t
                to[int(cache.table[i, pos // bt]), :, pos % bt] = y[at + t]
            at += n
    la.la_kv_write(cache.layer(), k, v, cu, torch.tensor(kv, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(cache.err) == 0
    assert torch.equal(cache.dev.cpu(), want)


def test_eight_bit_values_of_every_bf16():
    """Every bf16 value, NaN and infinities included, through an 8-bit cache of scale 1."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).reshape(1024, 1, 64).cuda()
    cache = torch.zeros((64, 2 * 16 * 64), dtype=torch.uint8, device="cuda")
    table = torch.arange(64, dtype=torch.int32, device="cuda")[None]
    layer = la.make_kv_layer(cache, table, 16, 1, 64, torch.float8_e4m3fn)
    la.la_kv_write(layer, x, x, torch.tensor([0, 1024], dtype=torch.int32, device="cuda"),
                   torch.tensor([1024], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    got = cache[:, :1024].cpu().view(torch.float8_e4m3fn).float().reshape(-1)
    f = bits.view(torch.bfloat16).float()
    want = f.clamp(-448, 448).to(torch.float8_e4m3fn).float()
    assert torch.equal(torch.isnan(got), torch.isnan(f))
    ok = ~torch.isnan(f)
    assert torch.equal(got[ok], want[ok])


def test_writes_outside_the_table_are_counted_and_left_out():
    gen = torch.Generator().manual_seed(52)
    cache = Cache(gen, [40, 40], 2, 128, "bf16", 16)
    cache.table[1, 1] = -1
    cache.table_dev.copy_(cache.table)
    before = cache.dev.clone()
    k = _rand(gen, 60, 2, 128).to(torch.bfloat16).cuda()
    # sequence 0: 30 tokens end at key 20 (ten below zero); sequence 1: 30 tokens end at key 60 (12 past the table)
    la.la_kv_write(cache.layer(), k, k, torch.tensor([0, 30, 60], dtype=torch.int32, device="cuda"),
                   torch.tensor([20, 60], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(cache.err) == 10 + 12 + 2            # and keys 30 and 31 in the missing block
    changed = (cache.dev != before).any(1).cpu()
    named = {int(b) for b in cache.table[0, :2]} | {int(cache.table[1, 2])}
    assert set(torch.nonzero(changed)[:, 0].tolist()) <= named
