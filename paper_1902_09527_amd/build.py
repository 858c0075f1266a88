"""Compile the HIP library ``libkmeans_mti.so`` for gfx950 (in-tree).

    python -m paper_1902_09527_amd.build

Every HIP source is compiled with packed float32 instructions disabled
(``-target-feature -packed-fp32-ops``); the host pass warns that it does not
know the feature, which is harmless.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libkmeans_mti.so")
SOURCES = [os.path.join(CSRC, "km_kernels.hip"), os.path.join(CSRC, "km_large.hip"),
           os.path.join(CSRC, "km_small.hip"), os.path.join(CSRC, "km_pp.hip"),
           os.path.join(CSRC, "km_gen.hip"),
           os.path.join(CSRC, "km_sort.hip"), os.path.join(CSRC, "km_norm.hip"),
           os.path.join(CSRC, "km_adapter.hip"),
           os.path.join(CSRC, "km_group.hip"), os.path.join(CSRC, "km_fp8.hip"),
           os.path.join(CSRC, "km_table.hip"), os.path.join(CSRC, "km_clip.hip"),
           os.path.join(CSRC, "km_ops.hip"),
           os.path.join(CSRC, "km_host.hip")]
ARCH = "gfx950"

HIPCC_FLAGS = [
    "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + INCLUDE, "-I" + CSRC,
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cand = os.path.join(rocm, "bin", "hipcc")
    return cand if os.path.exists(cand) else "hipcc"


def build(verbose: bool = False) -> str:
    """Compile every HIP source and link the shared library next to this file."""
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc()] + HIPCC_FLAGS + ["-shared", "-o", tmp] + SOURCES
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l and l.strip())
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err:
        print(err, file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
