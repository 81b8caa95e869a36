"""Builds libstarq.so (the HIP kernels and the C ABI) for gfx950 with hipcc.

Usage: ``python -m paper_2609_32814_amd.build`` or ``build()`` from Python.
Objects go to ``paper_2609_32814_amd/_build/``; the library is written next
to this file so that it travels with the source tree.
"""

from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libstarq.so")
SOURCES = ["plan.hip", "gemm.hip", "gemm_async.hip", "gemm_async_many.hip", "gemm_narrow.hip", "colsum.hip", "swiglu.hip", "decode.hip", "decode_stack.hip", "graph_fill.hip", "scratch.hip", "attention.hip", "attn_pack.hip", "attn_packed.hip", "attn_bwd.hip",
           "attn_paged.hip", "kv_pages.hip", "api.cpp"]
ARCH = "gfx950"

HIPCC_FLAGS = [
    "-x", "hip", f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-Wall", "-Wno-unused-function",
    # keep the compiler from forming packed fp32 VALU ops (v_pk_*_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found; the ROCm toolchain is required to build libstarq")


# Per-source flags.  The attention kernels keep their MFMA accumulators in
# VGPRs: the softmax works on every score, and accumulators in AGPRs would
# cost a v_accvgpr_read/write pair per value per step.  The small-tile GEMM
# does the same: its tiles are a few K steps long, so the epilogue's reads
# of the accumulators are a large share of its instructions.
EXTRA_FLAGS = {"attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "attn_packed.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "attn_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "attn_paged.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "gemm_narrow.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc(), *HIPCC_FLAGS, *EXTRA_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source and link libstarq.so.  Always rebuilds."""
    os.makedirs(BUILD, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(4, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
