"""Arguments of the attention and block entry points at the ends of their types,
refused before any launch.  Device pointers here are dummies that validation
never dereferences."""
import ctypes

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
