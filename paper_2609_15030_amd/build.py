"""Build the gfx950 shared library in-tree with hipcc.

``python -m paper_2609_15030_amd.build`` compiles csrc/linattn.hip (the
linear-attention path), csrc/attn.hip (attention over a cache and the
cache's blocks) and csrc/rope.hip (rotary positions), side by side, and links them into
paper_2609_15030_amd/liblinattn.so.  Every call compiles (no caching): the
output is written to a temporary name and moved into place.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRCS = [os.path.join(PKG, "csrc", f) for f in ("linattn.hip", "attn.hip", "rope.hip")]
LIB = os.path.join(PKG, "liblinattn.so")
ARCH = "gfx950"

HIPCC_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed fp32 VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA results in VGPRs: the scan's state feeds VALU converts and scales
    # every chunk, and AGPR results would cost a move per element and use
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    path = os.path.join(rocm, "bin", "hipcc")
    return path if os.path.exists(path) else "hipcc"


def _report(cmd, returncode, stderr, verbose):
    # hipcc's host pass does not know the packed-fp32 feature; drop that note
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in stderr.splitlines() if noise not in l)
    if returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)} failed ({returncode}):\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)


def build_library(verbose: bool = False) -> str:
    tmp = LIB + f".tmp{os.getpid()}"
    with tempfile.TemporaryDirectory() as d:
        objs = [os.path.join(d, os.path.basename(s) + ".o") for s in SRCS]
        cmds = [[hipcc(), *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), "-c", s,
                 "-o", o] for s, o in zip(SRCS, objs)]
        link = [hipcc(), f"--offload-arch={ARCH}", "-shared", *objs, "-o", tmp]
        if verbose:
            print("\n".join(" ".join(c) for c in [*cmds, link]), flush=True)
        procs = [subprocess.Popen(c, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True) for c in cmds]
        done = [p.communicate()[1] for p in procs]
        for c, p, err in zip(cmds, procs, done):
            _report(c, p.returncode, err, verbose)
        res = subprocess.run(link, capture_output=True, text=True)
        _report(link, res.returncode, res.stderr, verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
