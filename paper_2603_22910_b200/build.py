"""Builds libechokv.so (the C-ABI library) in-tree with nvcc for sm_100a.

    python -m paper_2603_22910_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libechokv.so")
SOURCES = ["echokv_host.cu", "simt_kernels.cu", "stored_mma.cu", "recon_tc.cu", "recon_pair.cu", "recon_quad.cu", "absorbed.cu", "prefill.cu", "noalloc.cu",
           "serving_host.cu", "plan.cu", "rotate.cu", "quant_append.cu", "quant_attn.cu", "quant_chunk.cu"]
HEADERS = ["common.cuh", "kernels.h", "recon_tc.h", "recon_common.cuh", "stored_mma.h", "absorbed.h", "prefill.h", "ptx_sm100.cuh",
           "serving.h", "quant_common.cuh", os.path.join("..", "..", "include", "echokv.h")]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source into one shared library; returns its path."""
    if not force and not needs_build():
        return LIB
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "--use_fast_math", "-t", "0", "-shared", "-Xcompiler", "-fPIC",
           "-cudart", "static", "-o", LIB]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed building libechokv.so")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
