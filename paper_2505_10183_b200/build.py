"""Builds the C-ABI CUDA library in-tree for sm_100a with nvcc, and the small Python module that passes
torch tensors to its training operators with the host compiler.  The module belongs to one torch and one Python;
the library does not, and is built and loaded without it where it cannot be built.

    python -m paper_2505_10183_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import importlib.util
import os
import re
import shutil
import subprocess
import sys
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
SOURCES = [os.path.join(_PKG, "csrc", "kaitian.cu"), os.path.join(_PKG, "csrc", "kt_host.cu"),
           os.path.join(_PKG, "csrc", "kt_rows.cu"),
           os.path.join(_PKG, "csrc", "kt_attn.cu"), os.path.join(_PKG, "csrc", "kt_embed.cu"),
           os.path.join(_PKG, "csrc", "kt_xent.cu"), os.path.join(_PKG, "csrc", "kt_orth.cu")]
DEPENDS = [os.path.join(_PKG, "csrc", "kt_kernels.cuh"), os.path.join(_PKG, "csrc", "kt_internal.h"),
           os.path.join(_PKG, "csrc", "kt_tensor.cuh"), os.path.join(_PKG, "csrc", "kt_pairs.cuh"),
           os.path.join(_PKG, "csrc", "kt_eight.cuh"), os.path.join(_PKG, "csrc", "kt_product.cuh")]
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


def _torch_folder() -> str:
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec is not None and spec.submodule_search_locations else ""


def torch_version() -> str:
    """The installed torch's version, without loading it ("" where there is none)."""
    try:
        with open(os.path.join(_torch_folder(), "version.py")) as f:
            return re.search(r"^__version__ = '(.*)'", f.read(), re.M).group(1)
    except (OSError, AttributeError):
        return ""


def fast_belongs() -> str:
    """What the operators' module is built for; the built file holds these words."""
    return "arguments of the operators, for torch %s and %s" % (torch_version(), sys.implementation.cache_tag)


def fast_is_of_another() -> bool:
    with open(FAST, "rb") as f:
        return fast_belongs().encode() not in f.read()


def can_build_fast() -> bool:
    """Whether there is a host compiler and the headers of torch and Python."""
    headers = (os.path.join(_torch_folder(), "include", "torch", "csrc", "autograd", "python_variable.h"), os.path.join(sysconfig.get_paths()["include"], "Python.h"))
    return shutil.which("g++") is not None and bool(torch_version()) and all(os.path.exists(h) for h in headers)


def _lib_is_stale() -> bool:
    return _older(LIB, SOURCES + DEPENDS + HEADERS)


def _fast_is_stale() -> bool:
    return _older(FAST, [FAST_SOURCE] + HEADERS) or fast_is_of_another()


def is_stale() -> bool:
    """Whether build() has something to do (the module counts only where it can be built)."""
    return _lib_is_stale() or (_fast_is_stale() and can_build_fast())


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
    torch = _torch_folder()
    cuda = os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda"
    includes = [os.path.join(torch, "include"), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", '-DKT_BELONGS="%s"' % fast_belongs()] + ["-I" + d for d in includes]
            + ["-o", out, FAST_SOURCE, "-L" + os.path.join(torch, "lib")]
            + ["-l" + n for n in ("torch_python", "torch_cpu", "c10", "c10_cuda")] + ["-Wl,-rpath," + os.path.join(torch, "lib")])


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _lib_is_stale():
        _run(lambda out: [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", out] + SOURCES, LIB, verbose)
    if force or _fast_is_stale():
        if can_build_fast():
            _run(_fast_command, FAST, verbose)
        else:
            sys.stderr.write("%s is not built: it needs g++ and the headers of torch and Python; the operators of a training step need it, "
                             "the rest of the library does not\n" % FAST)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
