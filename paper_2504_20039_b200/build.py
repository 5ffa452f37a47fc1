"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libaj_verify.so")
SOURCES = ["aj_api.cu", "aj_umma_vm.cu", "aj_umma_pair.cu", "aj_simt.cu", "aj_judge.cu", "aj_rank.cu", "aj_static.cu", "aj_lr.cu",
           "aj_kv_api.cu", "aj_kv_append.cu", "aj_kv_simt.cu", "aj_kv_few.cu", "aj_kv_umma.cu", "aj_kv_weigh.cu", "aj_kv_weigh_umma.cu", "aj_kv_evict.cu", "aj_kv_join.cu",
           "aj_score_api.cu", "aj_score_simt.cu", "aj_score_finish.cu", "aj_score_umma.cu", "aj_norm.cu"]
HEADERS = ["aj_internal.cuh", "aj_ptx.cuh", os.path.join("..", "..", "include", "aj_verify.h"),
           "aj_kv.cuh", "aj_kv_line.cuh", "aj_kv_mma.cuh", "aj_kv_tc.cuh", os.path.join("..", "..", "include", "aj_kv.h"),
           "aj_score.cuh", "aj_norm.cuh", os.path.join("..", "..", "include", "aj_score.h")]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC", "-cudart", "static", "--threads", "0",
]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libaj_verify.so next to this file; returns its path."""
    if force or _stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        tmp = f"{LIB}.{os.getpid()}.tmp"
        cmd = [nvcc, *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-o", tmp,
               *[os.path.join(CSRC, s) for s in SOURCES]]
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys

    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
