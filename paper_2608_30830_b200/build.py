"""Builds libkvr.so (CUDA kernels + C ABI) in-tree with nvcc for sm_100a."""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
SO = os.path.join(PKG, "libkvr.so")
SOURCES = ["kvr_kernels.cu", "kvr_engine.cu", "kvr_lib.cu", "kvr_noalloc.cu", "kvr_policy.cpp", "kvr_controller.cpp", "kvr_numa.cpp",
           "kvr_cache.cu", "kvr_pages.cu", "kvr_attend.cu", "kvr_attend_bf16.cu", "kvr_attend_f16.cu", "kvr_attend_e4m3.cu", "kvr_attend_int8.cu",
           "kvr_attend_e2m1.cu"]
DEPS = SOURCES + ["kvr_kernels.cuh", "kvr_cache.cuh", "kvr_pages.cuh", "kvr_attend.cuh", "kvr_attend_common.cuh",
                  "kvr_attend_rows.cuh", "kvr_attend_rows4.cuh", "kvr_attend_tiles.cuh", "kvr_meta.hpp", "kvr_numa.hpp", "kvr_once.hpp", "kvr_pool.hpp", os.path.join("..", "..", "include", "kvr.h")]


def stale():
    if not os.path.exists(SO):
        return True
    t = os.path.getmtime(SO)
    return any(os.path.getmtime(os.path.join(CSRC, d)) > t for d in DEPS)


def build(force=False, verbose=False):
    """Compile when sources are newer than the library.  Returns the path of libkvr.so."""
    if not (force or stale()):
        return SO
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = SO + ".%d.tmp" % os.getpid()
    flags = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
             "-Xcompiler", "-fPIC,-Wall", "-cudart", "static"] + (["-Xptxas=-v"] if verbose else [])
    with tempfile.TemporaryDirectory() as objects:
        def compile_one(source):
            out = os.path.join(objects, source + ".o")
            subprocess.check_call(flags + ["-c", "-o", out, os.path.join(CSRC, source)])
            return out

        with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as pool:
            parts = list(pool.map(compile_one, SOURCES))
        subprocess.check_call(flags + ["-shared", "-o", tmp] + parts)
    os.replace(tmp, SO)
    return SO


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
