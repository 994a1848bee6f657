"""In-tree build of the CUDA library (``libdvdq.so`` next to this file) with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libdvdq.so")
SOURCES = ["dvdq_lib.cu", "dvdq_block.cu", "dvdq_rows.cu", "dvdq_rows_bf16.cu", "dvdq_rows_f16.cu", "dvdq_rows_f32.cu",
           "dvdq_linear_int8.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return exe


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, d) for d in os.listdir(CSRC) if d.endswith((".cu", ".cuh"))]
    deps.append(os.path.join(os.path.dirname(_HERE), "include", "dvdq.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile the sources of ``csrc`` side by side and link ``libdvdq.so`` (cross-compiles without a GPU)."""
    if not force and not is_stale():
        return LIB_PATH
    tag = f".tmp{os.getpid()}"
    flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else [])
    objects = [os.path.join(_HERE, s + tag + ".o") for s in SOURCES]
    try:
        jobs = [subprocess.Popen([_nvcc(), *flags, "-c", "-o", o, os.path.join(CSRC, s)], cwd=CSRC)
                for s, o in zip(SOURCES, objects)]
        codes = [j.wait() for j in jobs]
        for s, code in zip(SOURCES, codes):
            if code != 0:
                raise subprocess.CalledProcessError(code, f"nvcc -c {s}")
        subprocess.run([_nvcc(), *flags, "-shared", "-o", LIB_PATH + tag, *objects, "-lcudart"], check=True, cwd=CSRC)
        os.replace(LIB_PATH + tag, LIB_PATH)
    finally:
        for o in objects:
            if os.path.exists(o):
                os.remove(o)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
