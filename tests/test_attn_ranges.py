"""Arguments of the attention and block entry points at the ends of their types,
refused before any launch.  Device pointers here are dummies that validation
never dereferences."""
import ctypes

import numpy as np
import pytest

from paper_2609_15030_amd import linattn as la

P = 0x10000                    # a 16-byte aligned address
LIB = la.library()


@pytest.mark.parametrize("max_blocks", [1 << 28, (1 << 59) + 40, 1 << 60, (1 << 63) - 1])
def test_tables_whose_tokens_pass_an_int64_are_refused(max_blocks):
    """1 << 60 blocks of 16 tokens are 2^64 tokens, which wraps to none."""
    y = la.LaKvLayer(P, 100, 65536, 0, 8192, 16, 2, 128, la.LA_BF16, 1.0, 1.0, P, max_blocks, None)
    assert LIB.la_kv_write(ctypes.byref(y), la.LA_BF16, P, 0, P, 0, P, 2, 10, P, None) == la.LA_ERR_INVALID_ARG
    s = la.make_attn_shape(2, 8, 2, 128)
    assert LIB.la_attn_decode(ctypes.byref(s), ctypes.byref(y), P, P, 0, None, P, P, 1 << 20, None) == la.LA_ERR_INVALID_ARG
    assert "max_blocks" in la.last_error_message()


def test_launches_past_2_to_32_threads_are_refused():
    """16.8 million row tiles, rows of a join, prefix tiles or table parts: more threads than a launch can have."""
    cu = np.arange(202, dtype=np.int32)
    s = la.make_attn_shape(201, 1 << 17, 1 << 17, 64)
    bad = la.LA_ERR_INVALID_ARG
    assert LIB.la_attn_prefill(ctypes.byref(s), P, P, P, P, cu.ctypes.data, P, P, 1 << 30, None) == bad
    y = la.LaKvLayer(P, 100, 1 << 30, 0, 1 << 29, 16, 1 << 17, 64, la.LA_BF16, 1.0, 1.0, P, 40, None)
    dec = lambda kv, g=None: LIB.la_attn_decode(ctypes.byref(s), ctypes.byref(y), P, P, kv, g, P, P, 1 << 62, None)
    assert dec(600) == bad
    groups = la.LaPrefixGroups(200, 1, P, P, 64)
    assert dec(64, ctypes.byref(groups)) == bad
    p = la.LaBlockPool(P, 100, 4096, 1 << 20, 1 << 13, 16, P, P, P, P, None)
    assert LIB.la_blocks_compact(ctypes.byref(p), None, P, 1 << 20, None) == bad
