"""Caches with a scale for each block and head, and reads of any cache, on the
CPU: what the entry points and the binding refuse before any launch.  Device
pointers here are dummies that validation never dereferences."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_15030_amd import linattn as la

P = 0x10000
LIB = la.library()
PART = 2 * 16 * 128                    # bytes of a layer's keys in a block


def _layer(dtype=la.LA_INT8_BLOCK, **kw):
    y = la.LaKvLayer(P, 100, 65536, 0, 8192, 16, 2, 128, dtype, 1.0, 1.0, P, 40, None, 16384, 16392)
    for k, v in kw.items():
        setattr(y, k, v)
    return y


def _write(y, io=la.LA_BF16):
    return LIB.la_kv_write(ctypes.byref(y), io, P, 0, P, 0, P, 2, 10, P, None)


def _read(y, io=la.LA_BF16, k=P, ks=0, v=P, seqs=2, toks=10, cu=P, kv=P):
    return LIB.la_kv_read(ctypes.byref(y), io, k, ks, v, 0, cu, seqs, toks, kv, None)


def _attend(y, io=la.LA_BF16):
    s = la.make_attn_shape(2, 8, 2, 128, io)
    cu, kv = np.array([0, 3, 9], np.int32), np.array([30, 600], np.int32)
    a = LIB.la_attn_prefill_paged(ctypes.byref(s), ctypes.byref(y), P, P, cu.ctypes.data, P, kv.ctypes.data, P, P, 1 << 30, None)
    b = LIB.la_attn_decode(ctypes.byref(s), ctypes.byref(y), P, P, 600, None, P, P, 1 << 40, None)
    assert a == b
    return a


@pytest.mark.parametrize("dtype", [la.LA_INT8_BLOCK, la.LA_FP8_E4M3_BLOCK])
@pytest.mark.parametrize("change", [
    dict(k_scales=-4), dict(k_scales=16385), dict(v_scales=16390), dict(k_scales=65532), dict(v_scales=65536),
    dict(v_scales=16388), dict(k_scales=16392), dict(k_scales=0), dict(v_scales=PART - 4), dict(k_scales=8192 + 64),
    dict(v_scales=8192 - 4, v_offset=8192, k_offset=16400), dict(k_scale=2.0), dict(v_scale=0.5), dict(v_offset=16384),
    dict(k_scales=(1 << 63) - 4), dict(dtype=5)], ids=str)
def test_layers_are_refused(dtype, change):
    if "dtype" not in change:
        change = dict(change, dtype=dtype)
    y = _layer(**change)
    if change.get("v_scales") == 8192 - 4 and "k_offset" in change:
        y.k_offset, y.k_scales = 16400, 32768         # the value scales reach into the values
    assert _write(y) == la.LA_ERR_INVALID_ARG
    assert _read(y) == la.LA_ERR_INVALID_ARG
    assert _attend(y) == la.LA_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [la.LA_INT8_BLOCK, la.LA_FP8_E4M3_BLOCK])
def test_codes_go_with_bf16(dtype):
    assert _write(_layer(dtype), la.LA_F32) == la.LA_ERR_UNSUPPORTED
    assert _attend(_layer(dtype), la.LA_F32) == la.LA_ERR_UNSUPPORTED


def test_reads_are_refused():
    bf16, f32 = _layer(la.LA_BF16, k_scales=0, v_scales=0), _layer(la.LA_F32, v_offset=16384)
    assert _read(f32) == la.LA_ERR_UNSUPPORTED
    for y in (bf16, _layer()):
        for kw in (dict(io=la.LA_FP8_E4M3), dict(k=None), dict(v=None), dict(cu=None), dict(kv=None), dict(k=P + 8),
                   dict(ks=100), dict(ks=257), dict(ks=1 << 25), dict(toks=-1), dict(toks=1 << 31), dict(seqs=-1)):
            assert _read(y, **kw) == la.LA_ERR_INVALID_ARG, kw
        assert _read(y, toks=0, k=None) == la.LA_OK and _read(y, seqs=0, cu=None) == la.LA_OK
    assert LIB.la_kv_read(None, la.LA_BF16, P, 0, P, 0, P, 2, 10, P, None) == la.LA_ERR_INVALID_ARG


def test_scales_of_other_types_are_not_read():
    """A caller built before the scales were there passes a shorter struct."""
    y = _layer(la.LA_BF16, k_scales=-1, v_scales=-1)
    assert LIB.la_kv_write(ctypes.byref(y), la.LA_BF16, P, 0, P, 0, P, 2, 0, P, None) == la.LA_OK


class _Cuda(torch.Tensor):
    """A CPU tensor that calls itself a device one, for checks that come before any use."""
    @property
    def is_cuda(self):
        return True


def _dev(t):
    return t.as_subclass(_Cuda)


def test_the_binding_names_types_by_their_scales():
    cache, table = _dev(torch.zeros((3, 65536), dtype=torch.uint8)), _dev(torch.zeros((1, 4), dtype=torch.int32))
    make = lambda dt, **kw: la.make_kv_layer(cache, table, 16, 2, 128, dt, **kw)
    assert make(torch.float8_e4m3fn).dtype == la.LA_FP8_E4M3
    y = make(torch.float8_e4m3fn, k_scales=16384)
    assert (y.dtype, y.k_scales, y.v_scales, y.v_offset) == (la.LA_FP8_E4M3_BLOCK, 16384, 16392, 4096)
    assert make(torch.int8, k_scales=16384, v_scales=32768).v_scales == 32768
    for dt, kw in ((torch.int8, {}), (torch.bfloat16, dict(k_scales=16384)), (torch.float8_e4m3fn, dict(v_scales=0)),
                   (torch.uint8, dict(k_scales=0)), (torch.float16, {})):
        with pytest.raises(ValueError):
            make(dt, **kw)


def test_the_binding_refuses_short_lists():
    cache, table = _dev(torch.zeros((3, 65536), dtype=torch.uint8)), _dev(torch.zeros((2, 4), dtype=torch.int32))
    y = la.make_kv_layer(cache, table, 16, 2, 128, torch.int8, k_scales=16384)
    k = _dev(torch.zeros((5, 2, 128), dtype=torch.bfloat16))
    i32 = lambda *v: _dev(torch.tensor(v, dtype=torch.int32))
    for cu, kv in ((i32(0, 1, 2, 5), i32(5, 5, 5)), (i32(0, 1, 5), i32(5))):
        with pytest.raises(ValueError):
            la.la_kv_read(y, k, k, cu, kv)
    with pytest.raises(ValueError):
        la.la_kv_read(y, k[:, :1], k, i32(0, 5), i32(5))
