"""Cache writes of some of a batch's sequences: offsets that begin behind the first
row and end before the last, against placing each row by its definition."""
import pytest
import torch

from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("cu,kv", [
    ([3, 10, 12], [30, 2]),
    ([5, 5, 6], [9, 40]),                            # an empty one first
    ([17, 17], [8]),                                 # nothing at all
    ([2] + [2 + i for i in range(1, 131)], [1 + i % 40 for i in range(130)]),      # three steps of 64 sequences
    ([1] + [1 + i // 3 for i in range(1, 200)], [5 + i % 30 for i in range(199)]),
])
def test_rows_outside_the_sequences_are_left_alone(cu, kv):
    bt, heads, d, n = 16, 2, 64, cu[-1] + 4
    width = 3
    gen = torch.Generator().manual_seed(91)
    x = torch.randn((n, 2 * heads, d), generator=gen).to(torch.bfloat16)
    table = torch.randperm(len(kv) * width, generator=gen).to(torch.int32).view(len(kv), width)
    want = torch.zeros((len(kv) * width, 2, heads, bt, d), dtype=torch.bfloat16)
    for i, L in enumerate(kv):
        for row in range(cu[i], cu[i + 1]):
            pos = L - (cu[i + 1] - row)
            for half in (0, 1):
                want[int(table[i, pos // bt]), half, :, pos % bt] = x[row, half * heads:(half + 1) * heads]
    cache = torch.zeros((len(kv) * width, want[0].numel() * 2), dtype=torch.uint8, device="cuda")
    err = _i32([0])
    layer = la.make_kv_layer(cache, table.cuda(), bt, heads, d, torch.bfloat16, err_count=err)
    y = x.cuda()
    la.la_kv_write(layer, y[:, :heads], y[:, heads:], _i32(cu), _i32(kv))
    torch.cuda.synchronize()
    assert int(err) == 0
    assert torch.equal(cache.cpu().view(torch.bfloat16).view(want.shape), want)
