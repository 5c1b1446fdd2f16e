"""Builds libqadc.so (the HIP kernels and the C ABI) in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqadc.so")
SOURCES = ["index.hip", "tables.hip", "quantize.hip", "scan.hip", "scan_mx.hip", "scan_mx_wide.hip", "ivf.hip", "coarse.hip", "coarse_half.hip", "encode.hip",
           "vec_lookup.hip", "vec_norm.hip", "vec_quantize.hip", "vec_matmul.hip", "vec_matmul_e4m3_e4m3.hip", "vec_matmul_e4m3_e5m2.hip",
           "vec_matmul_e5m2_e4m3.hip", "vec_matmul_e5m2_e5m2.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(CSRC, src.replace(".hip", ".o"))
    # the products with F32 scales multiply what the matrix instructions give, which can stay in vector registers for that
    more = ["-mllvm", "-amdgpu-mfma-vgpr-form=1"] if src.startswith("vec_matmul_") else []
    subprocess.check_call([HIPCC, *FLAGS, *more, "-c", os.path.join(CSRC, src), "-o", obj])
    return obj


def build(verbose: bool = True) -> str:
    """Compile every source (always, so a stale library is never kept) and link."""
    srcs = [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
