"""Registers and LDS of the kernels of block-scaled caches and rotary positions, from the
built library's notes: no scratch memory, and as many workgroups on a compute unit as
their launch rules and figures count on."""
import re

import pytest

from test_attn_kernel_resources import kernels               # noqa: F401  (the fixture)
from test_kernel_resources import workgroups_per_cu


def _mine(kernels, pattern):                                 # noqa: F811
    found = {n: k for n, k in kernels.items() if re.search(pattern, n)}
    assert found
    return found


def test_nothing_spills_to_memory(kernels):                  # noqa: F811
    mine = _mine(kernels, r"_code|kv_read_kernel|rope_kernel")
    assert len(mine) >= 30
    assert [n for n, k in mine.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]] == []


@pytest.mark.parametrize("pattern,least", [
    (r"attn_(wide|decode)_kernel.*_code", 2),
    (r"attn_decode_own_kernel", 3),                          # a grid of three a CU
    (r"kv_write_codes_kernel", 4),                           # 16 waves with 16 KB each in flight
    (r"kv_read_kernel", 7),
    (r"rope_kernel", 6),
])
def test_workgroups_that_share_a_cu(kernels, pattern, least):      # noqa: F811
    mine = {n: workgroups_per_cu(k) for n, k in _mine(kernels, pattern).items()}
    assert min(mine.values()) >= least, mine
