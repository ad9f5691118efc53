"""Builds the C-ABI CUDA library in-tree for sm_100a with nvcc.

    python -m paper_2505_10183_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
SOURCES = [os.path.join(_PKG, "csrc", "kaitian.cu"), os.path.join(_PKG, "csrc", "kt_host.cu"),
           os.path.join(_PKG, "csrc", "kt_rows.cu"),
           os.path.join(_PKG, "csrc", "kt_attn.cu")]
DEPENDS = [os.path.join(_PKG, "csrc", "kt_kernels.cuh"), os.path.join(_PKG, "csrc", "kt_internal.h"),
           os.path.join(_PKG, "csrc", "kt_tensor.cuh"), os.path.join(_PKG, "csrc", "kt_pairs.cuh")]
HEADERS = [os.path.join(_ROOT, "include", "kaitian.h")]
LIB = os.path.join(_PKG, "libkaitian_b200.so")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "--threads", "0"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > built for p in SOURCES + DEPENDS + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".%d.tmp" % os.getpid()
    cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout)
    if proc.returncode != 0:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError("nvcc failed (%d): %s" % (proc.returncode, " ".join(cmd)))
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
