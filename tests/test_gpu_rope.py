"""Rotary positions against the fp64 oracle (oracle/rope.py).

Bound of an output: a cosine or sine is off by at most 2.7e-7 (its angle by 1.5e-7: three
roundings of at most pi / 4, and 2^-32 turns; the polynomials by 2e-9 and two roundings),
the magnitude and the two products round it four times more, and the result rounds to its
type: magnitude (|x1| + |x2|) (2.7e-7 + 4 U32) + half an ulp."""
import numpy as np
import pytest
import torch

from oracle import rope as orope
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _check(y, x, pos, rope, dtype, transpose=False, magnitude=1.0):
    x, y = x.double().cpu().numpy(), y.double().cpu().numpy()
    want = orope.turn(x, pos, rope.frequencies, rope.layout, magnitude, transpose)
    r = rope.rotary_dim
    both = np.zeros_like(x)
    a = np.abs(x[..., :r])
    if rope.layout == "halves":
        s = a[..., :r // 2] + a[..., r // 2:]
        both[..., :r // 2] = both[..., r // 2:r] = s
    else:
        both[..., 0:r:2] = both[..., 1:r:2] = a[..., 0::2] + a[..., 1::2]
    half = 2.0 ** -8 if dtype == "bf16" else U32
    tol = abs(magnitude) * both * (2.7e-7 + 4 * U32) * 1.01 + half * 1.01 * np.abs(want) + 1e-37
    assert np.array_equal(y[..., r:], x[..., r:])
    worst = float(np.max((np.abs(y - want) / tol)[..., :r], initial=0.0))
    print(f"[rope] worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, worst


CASES = [
    # tokens, q heads, k heads, head dim, rotary dim, layout, type
    (1, 1, 1, 8, 2, "halves", "bf16"),
    (1, 4, 2, 64, 64, "halves", "f32"),
    (5, 8, 2, 128, 128, "halves", "bf16"),
    (7, 3, 1, 128, 64, "pairs", "bf16"),
    (130, 8, 8, 64, 48, "pairs", "f32"),
    (67, 6, 3, 80, 20, "halves", "bf16"),                      # halves of 10: values one by one at their ends
    (67, 6, 3, 80, 66, "halves", "f32"),
    (9, 2, 2, 128, 126, "pairs", "bf16"),
    (33, 40, 8, 256, 256, "halves", "bf16"),                   # several waves a token
    (12, 24, 8, 256, 254, "pairs", "f32"),
    (4, 2, 1, 512, 512, "halves", "f32"),
    (4, 2, 1, 1024, 512, "pairs", "bf16"),
    (3, 1, 130, 64, 32, "halves", "bf16"),
]


def _make(gen, T, heads, d, dtype, sliced):
    x = torch.randn((T, heads + (3 if sliced else 0), d), generator=gen).to(TYPES[dtype]).cuda()
    return x[:, :heads] if sliced else x


@pytest.mark.parametrize("sliced", [False, True], ids=["packed", "sliced"])
@pytest.mark.parametrize("transpose", [False, True], ids=["turn", "transposed"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_positions_given(case, transpose, sliced):
    T, hq, hk, d, r, layout, dtype = case
    gen = torch.Generator().manual_seed(51)
    rope = api.Rope(d, r, layout)
    q, k = _make(gen, T, hq, d, dtype, sliced), _make(gen, T, hk, d, dtype, sliced)
    pos = torch.randint(0, 5000, (T,), generator=gen).tolist()
    yq, yk = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    q0, k0 = q.clone(), k.clone()
    rope.apply(q, k, yq, yk, positions=_i32(pos), transpose=transpose)
    torch.cuda.synchronize()
    _check(yq, q0, pos, rope, dtype, transpose)
    _check(yk, k0, pos, rope, dtype, transpose)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    # in place: the same bits, and nothing beside the rows
    rope.apply(q, k, positions=_i32(pos), transpose=transpose)
    torch.cuda.synchronize()
    assert torch.equal(q, yq) and torch.equal(k, yk)


@pytest.mark.parametrize("sliced", [False, True], ids=["packed", "sliced"])
def test_what_lies_beside_the_rows_stays(sliced):
    gen = torch.Generator().manual_seed(52)
    x = torch.randn((6, 9, 128), generator=gen).to(torch.bfloat16).cuda()
    before = x.clone()
    rope = api.Rope(128, 96)
    rope.apply(x[:, 2:5], x[:, 6:8], positions=_i32(range(1, 7)))
    torch.cuda.synchronize()
    assert torch.equal(x[:, [0, 1, 5, 8]], before[:, [0, 1, 5, 8]])
    assert torch.equal(x[:, 2:8, 96:], before[:, 2:8, 96:]) and not torch.equal(x[:, 2:5, :96], before[:, 2:5, :96])


def test_positions_from_the_lengths():
    """Those of the keys that la_kv_write writes; rows outside every sequence stay, empty sequences have none."""
    gen = torch.Generator().manual_seed(53)
    new, kv, first = [5, 0, 1, 30] + [1] * 70, [900, 3, 1, 30] + list(range(1, 71)), 4
    T = first + sum(new) + 6
    cu = [first + sum(new[:i]) for i in range(len(new) + 1)]
    q, k = _make(gen, T, 4, 128, "bf16", True), _make(gen, T, 2, 128, "bf16", False)
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, kv)])
    yq, yk = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    rope = api.Rope(128)
    rope.apply(q, k, yq, yk, cu_seqlens=_i32(cu), kv_len=_i32(kv))
    torch.cuda.synchronize()
    rows = slice(first, first + sum(new))
    _check(yq[rows], q[rows], pos, rope, "bf16")
    _check(yk[rows], k[rows], pos, rope, "bf16")
    for y in (yq, yk):
        assert (y[:first] == 3.0).all() and (y[rows.stop:] == 3.0).all()


def test_thousands_of_sequences():
    gen = torch.Generator().manual_seed(59)
    new = torch.randint(-4, 4, (5000,), generator=gen).clamp(min=0)
    kv = new + torch.randint(0, 2000, (5000,), generator=gen)
    T = int(new.sum())
    cu = torch.cumsum(torch.cat([torch.zeros(1, dtype=torch.int64), new]), 0)
    pos = torch.cat([torch.arange(int(L - n), int(L)) for n, L in zip(new, kv)])
    x = _make(gen, T, 1, 64, "bf16", False)
    rope, y, z = api.Rope(64), torch.empty_like(x), torch.empty_like(x)
    rope.apply(x, None, y, cu_seqlens=cu.to(torch.int32).cuda(), kv_len=kv.to(torch.int32).cuda())
    rope.apply(x, None, z, positions=pos.to(torch.int32).cuda())
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    _check(z[-300:], x[-300:], pos[-300:].tolist(), rope, "bf16")


@pytest.mark.parametrize("scaling", [("linear", 4.0), ("base", 8.0), ("parts", 8.0, 4096.0, 1.0, 32.0)], ids=lambda s: s[0])
def test_far_positions_under_a_scaling(scaling):
    """Up to the ends of an int32, where an angle in fp32 would be none."""
    gen = torch.Generator().manual_seed(54)
    pos = [0, 1, 131071, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -1, -2 ** 31, 987654321]
    x = _make(gen, len(pos), 2, 64, "f32", False)
    magnitude = 0.1 * float(np.log(8.0)) + 1.0
    rope = api.Rope(64, 64, "pairs", 5e5, la.make_rope_scaling(*scaling), magnitude=magnitude)
    y, _ = rope.apply(None, x, k_out=torch.empty_like(x), positions=_i32(pos))[::-1]
    torch.cuda.synchronize()
    _check(y, x, pos, rope, "f32", magnitude=float(np.float32(magnitude)))


def test_given_frequencies():
    """Any finite ones: above a turn a token, negative, none."""
    gen = torch.Generator().manual_seed(55)
    x = _make(gen, 40, 2, 16, "f32", False)
    rope = api.Rope(16, 10, frequencies=np.array([0.0, 7.0, -0.3, 100.25, 1e-9]))
    y = torch.empty_like(x)
    rope.apply(x, None, y, positions=_i32(range(40)))
    torch.cuda.synchronize()
    _check(y, x, range(40), rope, "f32")


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_the_transposed_rotation_is_the_gradient(layout):
    """Against differences of a smooth loss in fp64 through the oracle, and <R x, g> = <x, R^T g>."""
    gen = torch.Generator().manual_seed(56)
    rope = api.Rope(16, 12, layout, magnitude=1.25)
    x, g = _make(gen, 3, 2, 16, "f32", False), _make(gen, 3, 2, 16, "f32", False)
    pos, dx = [3, 50, 7000], torch.empty_like(x)
    rope.apply(g, None, dx, positions=_i32(pos), transpose=True)
    torch.cuda.synchronize()
    x0, g0, got = x.double().cpu().numpy(), g.double().cpu().numpy(), dx.double().cpu().numpy()
    loss = lambda z: float(np.sum(g0 * orope.turn(z, pos, rope.frequencies, layout, 1.25)))
    h = 2.0 ** -10                                               # the loss is linear: differences are its slope
    for i in np.ndindex(*x0.shape):
        up, down = x0.copy(), x0.copy()
        up[i] += h
        down[i] -= h
        want = (loss(up) - loss(down)) / (2 * h)
        assert abs(got[i] - want) <= 1.25 * 2 * np.abs(g0).max() * (2.7e-7 + 5 * U32) + 1e-11, i


def test_infinities_and_nan_stay_in_their_pairs():
    rope = api.Rope(64, 48, "halves")
    x = torch.ones((4, 2, 64), device="cuda", dtype=torch.bfloat16)
    x[1, 0, 5], x[2, 1, 30], x[3, 0, 60] = float("nan"), float("inf"), float("nan")
    y = torch.empty_like(x)
    rope.apply(x, None, y, positions=_i32([9] * 4))
    torch.cuda.synchronize()
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 0, [5, 29]] = want[2, 1, [30, 6]] = True
    want[3, 0, 60] = True
    assert torch.equal(bad, want)


def test_no_tokens_and_either_rows_alone():
    rope = api.Rope(128)
    none = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    rope.apply(none, none[:, :2], positions=_i32([]))
    gen = torch.Generator().manual_seed(57)
    q, k = _make(gen, 6, 4, 128, "bf16", False), _make(gen, 6, 2, 128, "bf16", False)
    yq, yk, zq, zk = (torch.empty_like(t) for t in (q, k, q, k))
    pos = _i32(range(6))
    rope.apply(q, k, yq, yk, positions=pos)
    rope.apply(q, None, zq, positions=pos)
    rope.apply(None, k, None, zk, positions=pos)
    torch.cuda.synchronize()
    assert torch.equal(yq, zq) and torch.equal(yk, zk)


def test_captured_and_on_another_stream():
    gen = torch.Generator().manual_seed(58)
    rope = api.Rope(128)
    q, k = _make(gen, 3, 4, 128, "bf16", False), _make(gen, 3, 2, 128, "bf16", False)
    yq, yk = torch.empty_like(q), torch.empty_like(k)
    cu, kv = _i32([0, 1, 2, 3]), _i32([17, 5, 70])
    rope.apply(q, k, yq, yk, cu_seqlens=cu, kv_len=kv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rope.apply(q, k, yq, yk, cu_seqlens=cu, kv_len=kv)
    st = torch.cuda.Stream()
    for _ in range(3):
        kv += 1
        q.copy_(_make(gen, 3, 4, 128, "bf16", False))
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            zq, zk = rope.apply(q, k, torch.empty_like(q), torch.empty_like(k), cu_seqlens=cu, kv_len=kv)
        torch.cuda.synchronize()
        assert torch.equal(yq, zq) and torch.equal(yk, zk)


@pytest.mark.parametrize("bad", ["short positions", "both", "neither", "type", "heads", "tokens"])
def test_the_binding_refuses(bad):
    rope = api.Rope(128)
    q, k = (torch.zeros((4, n, 128), dtype=torch.bfloat16, device="cuda") for n in (4, 2))
    kw = dict(positions=_i32(range(4)))
    if bad == "short positions":
        kw["positions"] = _i32(range(3))
    if bad == "both":
        kw.update(cu_seqlens=_i32([0, 4]), kv_len=_i32([4]))
    if bad == "neither":
        kw = {}
    if bad == "type":
        k = k.float()
    if bad == "heads":
        q = q.transpose(1, 2)
    if bad == "tokens":
        k = k[:3]
    with pytest.raises(ValueError):
        rope.apply(q, k, **kw)
    with pytest.raises(ValueError):
        rope.apply(None, None, positions=_i32([]))
