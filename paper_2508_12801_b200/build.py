"""Build libmaxscore.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmaxscore.so")
SOURCES = ["maxscore_api.cu", "blocks_api.cu", "topk_api.cu", "experts8_api.cu"]
HEADERS = ["common.cuh", "context.cuh", "tc.cuh", "flow.cuh", "gate.cuh", "move.cuh", "softtopk.cuh", "reroute.cuh", "alg1.cuh", "expert.cuh",
           "expert_tc.cuh", "expert_few.cuh", "expert_launch.cuh", "int8.cuh", "rows8.cuh", "norm.cuh", "topk.cuh",
           os.path.join("..", "..", "include", "maxscore.h")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-shared", "-Xcompiler", "-fPIC", "--cudart", "static", "--threads", str(len(SOURCES)), "-o", tmp]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += os.environ.get("MAXSCORE_NVCC_FLAGS", "").split()
    cmd += [os.path.join(CSRC, f) for f in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
