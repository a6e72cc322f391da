"""Builds libxkv.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libxkv.so")
SOURCES = ["xkv_api.cu", "xkv_score.cu", "xkv_score_tc.cu", "xkv_score_fused.cu", "xkv_select.cu", "xkv_decode.cu", "xkv_prefill.cu",
           "xkv_serve.cu", "xkv_decode_e4m3.cu", "xkv_pages.cu",
           "xkv_diff_prefill.cu", "xkv_diff_decode.cu"]
HEADERS = ["common.cuh", "ops.h", "score_params.h", "tc_common.cuh", "e4m3.cuh", os.path.join("..", "..", "include", "xkv.h")]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; libxkv.so cannot be built")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    return any(os.path.getmtime(p) > built for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source into paper_2412_05896_b200/libxkv.so; returns its path."""
    if not force and not is_stale():
        return LIB
    cmd = [_nvcc(), "--threads", "0", "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-Xcompiler", "-fPIC", "-shared", "-o", LIB]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, f) for f in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose:
        sys.stderr.write(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
