"""Builds the HIP library ``libnm_hip.so`` for gfx950 in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libnm_hip.so")
SOURCES = ["nm_tables.cpp", "nm_rows.hip", "nm_gemm.hip", "nm_gemm_direct.hip", "nm_gemm_end.hip", "nm_gemm_long.hip", "nm_gemm_unaligned.hip", "nm_gemm_ln.hip", "nm_qkv_attention.hip", "nm_attention.hip", "nm_block.hip", "nm_conv_chain.hip", "nm_conv_taps.hip", "nm_conv.hip",
           "nm_page_plan.hip", "nm_qk_rope.hip", "nm_paged_attention.hip", "nm_gemv_w4.hip", "nm_gemv_w4_bf16.hip",
           "nm_gemv_w4_f16.hip", "nm_layer.cpp"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
    # the fp32 epilogue is bit-reproducible: no implicit fused multiply-adds, no flushed denormals
    "-ffp-contract=off", "-fno-gpu-flush-denormals-to-zero",
    # packed fp32 instructions are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
    "-I", INCLUDE, "-I", CSRC,
]


def build_library(verbose: bool = False) -> str:
    """Compile every source for gfx950 and link the shared library.  Always recompiles."""
    objs = []

    def compile_one(src):
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0 or verbose:
            print(" ".join(cmd))
            print(r.stdout, r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}")
        return obj

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        print(r.stdout, r.stderr)
        raise RuntimeError("link failed")
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
