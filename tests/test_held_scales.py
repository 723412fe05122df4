"""The scale that a later write finds in its block: one past what any write can leave (the
scale of values of 2^127) is none, and counts as the least."""
import numpy as np
import pytest
import torch

from codes import CodeCache
from oracle import kv_codes as kc
from paper_2609_15030_amd import linattn as la

KINDS = ["e4m3", "int8"]
# the largest scale that a write can leave, and the next one of as many bits
LARGEST = {"e4m3": (2.0 ** 119, 2.0 ** 120), "int8": (130 * 2.0 ** 113, 131 * 2.0 ** 113)}


@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_scale(kind):
    most, next_one = LARGEST[kind]
    assert kc.scale_of(2.0 ** 127, kind) == most and kc.held(most, kind) == most
    for s in (next_one, 2.0 ** 121, 2.0 ** 126, 2.0 ** 127):
        assert kc.held(s, kind) == float(kc.LEAST)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_writes_behind_scales_past_the_largest(kind):
    """Ordinary tokens into blocks that hold such a scale keep their values; the largest possible one stays."""
    gen = torch.Generator().manual_seed(73)
    most, next_one = LARGEST[kind]
    held = [most, next_one, 2.0 ** 121, 2.0 ** 125, 2.0 ** 126, 2.0 ** 127]
    n = len(held)
    c = CodeCache(gen, kind, 1, 64, 16, np.arange(n, dtype=np.int32)[:, None], n)
    for half in (0, 1):
        code, scale = c.numbers(half)
        scale[:, 0] = held
        c.put(half, code, scale)
    c.dev.copy_(c.bytes)
    k, v = (torch.randn((n, 1, 64), generator=gen).to(torch.bfloat16).cuda() for _ in (0, 1))
    i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device="cuda")
    la.la_kv_write(c.layer(), k, v, i32(range(n + 1)), i32([9] * n))
    c.write(k, v, range(n + 1), [9] * n)
    torch.cuda.synchronize()
    c.same(kind)
    for half, x in ((0, k), (1, v)):
        code, scale = c.numbers(half)
        assert scale[0, 0] == most and np.all(scale[1:, 0] < 1.0)
        off = np.abs(code[1:, 0, 8] * scale[1:] - x[1:, 0].double().cpu().numpy())
        assert np.all(off <= np.maximum(2.0 ** -4 * np.abs(x[1:, 0].double().cpu().numpy()), scale[1:]))
