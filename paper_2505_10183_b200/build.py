"""Builds the C-ABI CUDA library in-tree for sm_100a with nvcc, and the small Python module that passes
torch tensors to its training operators with the host compiler.

    python -m paper_2505_10183_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
SOURCES = [os.path.join(_PKG, "csrc", "kaitian.cu"), os.path.join(_PKG, "csrc", "kt_host.cu"),
           os.path.join(_PKG, "csrc", "kt_rows.cu"),
           os.path.join(_PKG, "csrc", "kt_attn.cu")]
DEPENDS = [os.path.join(_PKG, "csrc", "kt_kernels.cuh"), os.path.join(_PKG, "csrc", "kt_internal.h"),
           os.path.join(_PKG, "csrc", "kt_tensor.cuh"), os.path.join(_PKG, "csrc", "kt_pairs.cuh")]
HEADERS = [os.path.join(_ROOT, "include", "kaitian.h")]
LIB = os.path.join(_PKG, "libkaitian_b200.so")
FAST_SOURCE = os.path.join(_PKG, "csrc", "kt_fast.cpp")
FAST = os.path.join(_PKG, "_fast.so")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "--threads", "0"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _older(target: str, sources) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(p) > os.path.getmtime(target) for p in sources)


def is_stale() -> bool:
    return _older(LIB, SOURCES + DEPENDS + HEADERS) or _older(FAST, [FAST_SOURCE] + HEADERS)


def _run(cmd, target: str, verbose: bool) -> None:
    """Runs a compiler whose output goes to a file beside `target`, which it replaces in one step."""
    tmp = target + ".%d.tmp" % os.getpid()
    proc = subprocess.run(cmd(tmp), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout)
    if proc.returncode != 0:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError("compiler failed (%d): %s" % (proc.returncode, " ".join(cmd(tmp))))
    os.replace(tmp, target)


def _fast_command(out: str):
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.submodule_search_locations:
        raise RuntimeError("torch is not installed: its headers are needed to build %s" % FAST)
    torch = spec.submodule_search_locations[0]
    cuda = os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda"
    includes = [os.path.join(torch, "include"), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared"] + ["-I" + d for d in includes] + ["-o", out, FAST_SOURCE, "-L" + os.path.join(torch, "lib")]
            + ["-l" + n for n in ("torch_python", "torch_cpu", "c10", "c10_cuda")] + ["-Wl,-rpath," + os.path.join(torch, "lib")])


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _older(LIB, SOURCES + DEPENDS + HEADERS):
        _run(lambda out: [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", out] + SOURCES, LIB, verbose)
    if force or _older(FAST, [FAST_SOURCE] + HEADERS):
        _run(_fast_command, FAST, verbose)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
