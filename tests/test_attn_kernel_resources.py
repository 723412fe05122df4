"""Registers, LDS and spills of the attention and block kernels, from the notes of
every code object in the built library: what their launch rules count on for
workgroups sharing a compute unit."""
import re
import struct
import subprocess

import pytest
import yaml

from paper_2609_15030_amd.build import LIB

from test_kernel_resources import workgroups_per_cu

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{demangled name without arguments: metadata} of all gfx950 code objects."""
    blob = open(LIB, "rb").read()
    found, at, folder = {}, blob.find(MAGIC), tmp_path_factory.mktemp("co")
    while at >= 0:
        n, = struct.unpack_from("<Q", blob, at + 24)
        pos = at + 32
        for _ in range(n):
            off, size, tlen = struct.unpack_from("<QQQ", blob, pos)
            if b"gfx950" in blob[pos + 24:pos + 24 + tlen]:
                path = folder / f"{at}.co"
                path.write_bytes(blob[at + off:at + off + size])
                notes = subprocess.run(["/opt/rocm/llvm/bin/llvm-readelf", "--notes", str(path)], check=True,
                                       capture_output=True, text=True).stdout
                meta = yaml.safe_load(notes[notes.index("---"):notes.index("...")]).get("amdhsa.kernels", [])
                names = subprocess.run(["c++filt"], input="\n".join(k[".name"] for k in meta), check=True,
                                       capture_output=True, text=True).stdout.split("\n")
                for s, k in zip(names, meta):
                    found[re.sub(r"^(void )?la::", "", s.split("(")[0])] = k
            pos += 24 + tlen
        at = blob.find(MAGIC, at + 1)
    return found


def test_both_halves_of_the_library_are_seen(kernels):
    assert any(n.startswith("gdr_") for n in kernels) and any(n.startswith("attn_") for n in kernels)


def test_nothing_spills_to_memory(kernels):
    """Scratch would put the inner loops' registers in memory."""
    mine = {n: k for n, k in kernels.items() if re.match(r"attn_|kv_write|blocks_|fork|extend|free_|compact", n)}
    assert len(mine) >= 25
    assert [n for n, k in mine.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]] == []


@pytest.mark.parametrize("pattern,least", [
    (r"attn_wide_kernel<", 2),               # one workgroup's loads hide behind the other's products
    (r"attn_decode_kernel<", 2),             # a grid of two a CU for the own keys
    (r"attn_tile_kernel<64, ", 4),           # a split call counts on four at 64 dims, two at 128
    (r"attn_tile_kernel<128, ", 2),
])
def test_workgroups_that_share_a_cu(kernels, pattern, least):
    mine = {n: workgroups_per_cu(k) for n, k in kernels.items() if n.startswith(pattern)}
    assert mine and min(mine.values()) >= least, mine
