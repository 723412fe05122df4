"""la_kv_read of an e4m3 cache with one scale: each value, code times an fp32 scale of 24
bits, is rounded once.  Compared with the product in fp64, where it is exact (28 bits)."""
import numpy as np
import pytest
import torch

from oracle import kv_codes as kc
from paper_2609_15030_amd import linattn as la

CODES = torch.arange(256, dtype=torch.uint8)
VALUES = CODES.view(torch.float8_e4m3fn).float().double().numpy()


def _twice(x):
    """The products as fp32 and then as bf16."""
    with np.errstate(over="ignore"):
        return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()


def _scales():
    """Scales at which two roundings differ from one for some code, and a few others: with some
    code the product is near a tie between two bf16 values, in the ordinary range, at its lower end and among the subnormals."""
    rng = np.random.default_rng(71)
    ties = 1 + (2 * np.arange(128) + 1) / 256
    near = (ties[:, None] / (1 + np.arange(1, 8) / 8)).astype(np.float32).ravel()
    near = np.concatenate([near * np.float32(2.0 ** e) for e in (-9, 0, 6, -120)])
    low = (2.0 ** rng.uniform(-131, -118, 150000)).astype(np.float32)
    some = []
    for s, least in ((near, 400), (low, 40)):
        x = kc.E4M3[None, :] * s.astype(np.float64)[:, None]
        differ = s[np.any(_twice(x) != kc.bf16(x), axis=1)]
        assert differ.size >= least
        some += differ[::max(1, differ.size // 60)].tolist()
    return some + [0.7065972089767456, 0.9131944179534912, 1.0, 0.37, 2.0 ** -149, 3e38, 7.59e35, 2.0 ** 119] + [1.0] * (len(some) % 2)


def test_one_rounding_to_bf16():
    """The oracle's against torch's, for values of fp32."""
    rng = np.random.default_rng(72)
    x = np.concatenate([2.0 ** rng.uniform(-149, 128, 4000) * rng.choice([-1, 1], 4000), [0.0, 1.0, 3.39e38, 2.0 ** -134, 3 * 2.0 ** -134]])
    x = x.astype(np.float32)
    tie = ((x.view(np.uint32) & np.uint32(0xFFFF0000)) | np.uint32(0x8000)).view(np.float32)
    for y in (x, tie):
        assert np.array_equal(kc.bf16(y), torch.from_numpy(y).to(torch.bfloat16).double().numpy())
    # off a tie by less than fp32 holds
    assert kc.bf16([1 + 2.0 ** -8 + 2.0 ** -40])[0] == 1 + 2.0 ** -7 and kc.bf16([1 + 2.0 ** -8])[0] == 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_one_scale_reads_round_once(out):
    d, bt = 64, 16
    cache = torch.zeros((1, 2 * bt * d), dtype=torch.uint8)
    cache[0, :256] = cache[0, bt * d:bt * d + 256] = CODES
    cache = cache.cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, cu, kv = i32(0).view(1, 1), i32(0, 4), i32(4)
    scales = _scales()
    for ks, vs in zip(scales[::2], scales[1::2]):
        layer = la.make_kv_layer(cache, table, bt, 1, d, torch.float8_e4m3fn, k_scale=ks, v_scale=vs)
        k, v = (torch.empty((4, 1, d), dtype=out, device="cuda") for _ in (0, 1))
        la.la_kv_read(layer, k, v, cu, kv)
        torch.cuda.synchronize()
        for y, s in ((k, ks), (v, vs)):
            x = VALUES * float(np.float32(s))
            with np.errstate(over="ignore"):
                want = kc.bf16(x) if out is torch.bfloat16 else x.astype(np.float32).astype(np.float64)
            assert np.array_equal(y.double().cpu().numpy().ravel(), want, equal_nan=True), s
