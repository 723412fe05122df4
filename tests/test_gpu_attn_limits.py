"""Attention at the ends of what the entry points accept: layers, lengths and
launches whose offsets pass 32 bits.  References are fp64 (oracle/attention.py)
with its derived bound."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _check(o, q, k, v, first, d, bf16, what):
    """o, q [n, heads, d] at positions first, ...; k, v [L, heads, d]."""
    ref, mean, size = oa.attend(_host(q), _host(k), _host(v), first, float(np.float32(d ** -0.5)))
    off = np.abs(_host(o) - ref) / oa.tolerance(ref, mean, size, k.shape[0], d, bf16)
    print(f"[attn limits] {what}: worst {off.max():.3f} of the bound", flush=True)
    assert off.max() <= 1.0, what


@pytest.mark.parametrize("kind,heads", [("f32", 16400), ("bf16", 32800)])
def test_a_layer_whose_keys_take_over_2_gb_of_a_block(kind, heads):
    """The last heads of a block begin past 2^31 bytes behind its keys."""
    d, bt, n, t = 128, 256, 3, TYPES[kind]
    part = heads * bt * d * torch.empty(0, dtype=t).element_size()
    assert part > 1 << 31
    cache = torch.empty((1, 2 * part), dtype=torch.uint8, device="cuda")
    layer = la.make_kv_layer(cache, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), bt, heads, d, t)
    gen = torch.Generator(device="cuda").manual_seed(61)
    q, k, v = (torch.randn((n, heads, d), generator=gen, device="cuda").to(t) for _ in range(3))
    kv = torch.tensor([n], dtype=torch.int32, device="cuda")
    la.la_kv_write(layer, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), kv)
    want = api.AttnPrefill(heads, heads, d, [n], dtype=t).run(q, k, v)
    got = api.AttnPrefill(heads, heads, d, [n], [n], dtype=t).run_paged(layer, q)
    one = api.AttnDecode(1, heads, heads, d, n, dtype=t).run(layer, q[n - 1:], kv)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    some = [0, heads // 2, heads - 17, heads - 16, heads - 1]
    x = [y[:, some] for y in (q, k, v)]
    _check(got[:, some], *x, 0, d, kind == "bf16", f"{heads} heads, prompt")
    _check(one[:, some], x[0][n - 1:], *x[1:], n - 1, d, kind == "bf16", f"{heads} heads, single token")
