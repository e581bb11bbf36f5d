"""Builds ``libisv.so`` in-tree with nvcc for sm_100a.

``python -m paper_2504_11816_b200.build`` (or :func:`build`) compiles the CUDA
sources under ``csrc/`` into ``paper_2504_11816_b200/libisv.so``.  nvcc
cross-compiles, so no GPU is needed to build.
"""
from __future__ import annotations

import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libisv.so")
SOURCES = ["isv_kernels.cu", "isv_api.cu", "isv_static.cu", "isv_linear.cu", "isv_q8.cu", "isv_q8_attn.cu", "isv_pages.cu",
           "isv_linear4.cu", "isv_chunk.cu", "isv_chunk_attn_64.cu", "isv_chunk_attn_80.cu", "isv_chunk_attn_128.cu", "isv_draft.cu"]
HEADERS = ["isv_kernels.cuh", "isv_q8.cuh", "isv_chunk.cuh", "isv_chunk_attn.cuh", "isv_host.hpp", os.path.join("..", "..", "include", "isv.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile what is out of date and link the shared library; returns its path."""
    headers = [os.path.join(CSRC, h) for h in HEADERS]
    objs = []
    procs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(CSRC, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + headers):
            cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
            procs.append((cmd, subprocess.Popen(cmd)))
    for cmd, p in procs:
        if p.wait() != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    if force or procs or _stale(LIB, objs):
        cmd = [_nvcc(), "-shared"] + NVCC_FLAGS[:2] + ["-o", LIB] + objs
        subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
