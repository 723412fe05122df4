"""The binding's structs lie in memory as the header's do: sizes and offsets from a C
program compiled against include/linattn.h."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_15030_amd import linattn as la

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"la_shape": la.LaShape, "la_attn_shape": la.LaAttnShape, "la_kv_layer": la.LaKvLayer,
           "la_prefix_groups": la.LaPrefixGroups, "la_block_pool": la.LaBlockPool, "la_kv_blocks": la.LaKvBlocks,
           "la_rope_scaling": la.LaRopeScaling, "la_rope_plan": la.LaRopePlan, "la_rope_rows": la.LaRopeRows,
           "la_rope_positions": la.LaRopePositions}


@pytest.fixture(scope="module")
def layout(tmp_path_factory):
    folder = tmp_path_factory.mktemp("abi")
    lines = ["#include <stdio.h>", '#include "linattn.h"', "int main(void) {"]
    for name, s in STRUCTS.items():
        lines.append(f'    printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'    printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in s._fields_]
    (folder / "abi.c").write_text("\n".join(lines + ["    return 0;", "}"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(folder / "abi.c"), "-o",
                    str(folder / "abi")], check=True)
    out = subprocess.run([str(folder / "abi")], check=True, capture_output=True, text=True).stdout
    return dict(line.split() for line in out.splitlines())


@pytest.mark.parametrize("name", STRUCTS)
def test_structs_match_the_header(layout, name):
    s = STRUCTS[name]
    assert int(layout[name]) == ctypes.sizeof(s)
    for f in s._fields_:
        assert int(layout[f"{name}.{f[0]}"]) == getattr(s, f[0]).offset, f[0]


def test_a_layer_without_scales_is_the_layer_that_was(layout):
    """The scales came behind everything else: callers of the other types may pass the struct without them."""
    assert int(layout["la_kv_layer.k_scales"]) == int(layout["la_kv_layer.err_count"]) + ctypes.sizeof(ctypes.c_void_p)
