"""Compile the CUDA library in-tree for sm_100a (nvcc cross-compiles without a GPU)."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libalexnet_b200.so")
LIB_TIMELINE = os.path.join(HERE, "libalexnet_b200_timeline.so")      # the same sources with -DALEXNET_TIMELINE
OBJECTS = os.path.join(HERE, "_build")
SOURCES = ["alexnet_api.cu", "operators.cu", "loader.cpp"]
TIMELINE_SOURCES = ["alexnet_api.cu"]
HEADERS = ["ptx.cuh", "tc_gemm.cuh", "kernels.cuh", "checkpoint.cuh", "group_norm.cuh", "linear_grad.cuh", os.path.join("..", "..", "include", "alexnet.h")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def _compile(source: str, flags: list) -> str:
    """One source to an object under _build/; the objects of different flags lie beside one another."""
    obj = os.path.join(OBJECTS, os.path.splitext(source)[0] + ("_timeline.o" if "-DALEXNET_TIMELINE" in flags else ".o"))
    subprocess.check_call(flags + ["-c", "-o", obj, os.path.join(CSRC, source)])
    return obj


def build(force: bool = False, verbose: bool = False, timeline: bool = False) -> str:
    """timeline=True builds the instrumented variant (per-role timers inside conv_kernel) as a second library."""
    lib = LIB_TIMELINE if timeline else LIB
    if not force and not timeline and not _stale():
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    # (No -split-compile: it cuts a file into parts to compile them side by side, and where it cuts changes the registers and spills of kernels whose
    # source did not change.  With it a training step of 128 images took 1.064 ms for 1.025.)
    flags = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-pthread"]
    if verbose:
        flags.append("-Xptxas=-v")
    os.makedirs(OBJECTS, exist_ok=True)
    jobs = [(src, flags + ["-DALEXNET_TIMELINE"] if timeline and src in TIMELINE_SOURCES else flags) for src in SOURCES]
    if timeline and not _stale():           # the library's own objects of the sources that have no timers
        jobs = [(src, f) for src, f in jobs if src in TIMELINE_SOURCES or not os.path.exists(os.path.join(OBJECTS, os.path.splitext(src)[0] + ".o"))]
    with concurrent.futures.ThreadPoolExecutor() as pool:
        list(pool.map(lambda job: _compile(*job), jobs))
    objects = [os.path.join(OBJECTS, os.path.splitext(src)[0] + ("_timeline.o" if timeline and src in TIMELINE_SOURCES else ".o")) for src in SOURCES]
    subprocess.check_call(flags + ["-shared", "-o", lib] + objects)
    return lib


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="--quiet" not in sys.argv, timeline="--timeline" in sys.argv))
