"""The oracle of block-scaled caches against torch's own e4m3 type, brute force
and the bounds that the scales are there for."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import kv_codes as kc


def test_e4m3_rounds_as_torch_does():
    all_codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    finite = all_codes[torch.isfinite(all_codes)].double().numpy()
    assert np.array_equal(kc.e4m3(finite), finite)
    mid = np.unique(np.abs(finite))
    x = np.concatenate([(mid[1:] + mid[:-1]) / 2, mid[:-1] * (2 / 3) + mid[1:] / 3, np.linspace(-448, 448, 4001)])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).float().double().numpy()
    assert np.array_equal(kc.e4m3(x.astype(np.float32)), want)


@pytest.mark.parametrize("kind,most", [("e4m3", 448), ("int8", 127)])
def test_scales_hold_their_values_and_are_the_least_that_do(kind, most):
    rng = np.random.default_rng(3)
    for a in np.concatenate([[0.0, 1.0, 127.0, 448.0, 449.0, 2.0 ** 127, 2.0 ** -110], 2.0 ** rng.uniform(-60, 60, 300)]):
        a = float(torch.tensor(a).to(torch.bfloat16))
        s = Fraction(kc.scale_of(a, kind))
        assert Fraction(a) <= most * s
        if s == Fraction(1, 2 ** 100):
            continue
        less = s / 2 if kind == "e4m3" else s * (1 - Fraction(1, 128))
        assert Fraction(a) > most * less
        assert kc.held(float(s), kind) == float(s)


@pytest.mark.parametrize("kind,half", [("e4m3", 0.0625), ("int8", None)])
def test_written_values_are_near_theirs(kind, half):
    """Each value is off by at most half a step: of its own (e4m3: 2^-4 of it, and
    2^-10 scales below the smallest normal), or of the scale; a scale that grew may
    add half a step each time."""
    rng = np.random.default_rng(5)
    H, bt, d, T = 2, 16, 8, 41
    x = torch.from_numpy(rng.normal(size=(T, H, d)) * 2.0 ** rng.integers(-3, 4, (T, 1, 1))).to(torch.bfloat16).double().numpy()
    table = np.array([[2, 0, 3]])
    code, scale = np.zeros((4, H, bt, d)), np.full((4, H), np.nan)
    at = 0
    for n in (1, 3, 17, 1, 19):
        kc.write(code, scale, table, bt, kind, x, [at, at + n], [at + n])
        at += n
    assert at == T
    for p in range(T):
        b = table[0][p // bt]
        s = scale[b][:, None]
        got = code[b, :, p % bt] * s
        bound = 5 * 0.5 * s if kind == "int8" else np.maximum(half * np.abs(x[p]), 5 * 2.0 ** -10 * s)
        assert np.all(np.abs(got - x[p]) <= bound * (1 + 1e-9))


def test_one_write_of_a_block_forgets_its_past():
    code, scale = np.full((1, 1, 16, 8), 7.0), np.full((1, 1), 1e9)
    kc.write(code, scale, np.array([[0]]), 16, "int8", np.ones((3, 1, 8)), [0, 3], [3])
    assert np.all(code[0, 0, :3] * scale[0, 0] > 0.99) and np.all(code[0, 0, 3:] == 7.0)
    # ... and one behind its first token does not
    kc.write(code, scale, np.array([[0]]), 16, "int8", np.full((1, 1, 8), 0.5), [0, 1], [4])
    assert scale[0, 0] == kc.scale_of(1.0, "int8")
