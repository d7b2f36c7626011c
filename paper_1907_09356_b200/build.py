"""Builds libchoco.so (the CUDA library behind the C interface) in-tree with nvcc."""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libchoco.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-fmad=false",                      # no fused multiply-add: results must be reproducible
    "-diag-suppress=186",               # "pointless comparison" in template branches that are compiled out
    "-Xcompiler", "-fPIC",
]


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h"))
    deps.append(os.path.join(HERE, "..", "include", "choco.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Every file by an nvcc of its own, side by side, then one link."""
    if force or stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        with tempfile.TemporaryDirectory() as objects:
            pairs = [(src, os.path.join(objects, os.path.basename(src) + ".o")) for src in sources()]

            def compile_one(pair):
                subprocess.check_call([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", pair[1], pair[0]])

            with concurrent.futures.ThreadPoolExecutor(max_workers=min(len(pairs), os.cpu_count() or 1)) as pool:
                list(pool.map(compile_one, pairs))
            subprocess.check_call([nvcc] + NVCC_FLAGS + ["-shared", "-o", LIB] + [obj for _, obj in pairs])
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
