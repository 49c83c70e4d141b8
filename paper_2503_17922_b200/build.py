"""Builds the C-ABI shared library (libwkv.so) in-tree with nvcc for sm_100a.

    python -m paper_2503_17922_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libwkv.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC",
]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    flags = [_nvcc()] + NVCC_FLAGS + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    # one compiler per source, as many at a time as there are cores
    objects = tempfile.mkdtemp(prefix="wkv-build-")
    try:
        def compile_one(src: str) -> str:
            obj = os.path.join(objects, os.path.basename(src) + ".o")
            subprocess.check_call(flags + ["-c", "-o", obj, src])
            return obj
        with ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as pool:
            objs = list(pool.map(compile_one, sources()))
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.check_call([_nvcc()] + NVCC_FLAGS[:2] + ["-shared", "-cudart", "static", "-o", tmp] + objs + ["-ldl"])
        os.replace(tmp, LIB)
    finally:
        shutil.rmtree(objects, ignore_errors=True)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
