"""Builds the CUDA library in-tree with nvcc for sm_100a, and the marshalling module beside it.

    python -m paper_2407_11062_b200.build
"""
from __future__ import annotations

import importlib.metadata
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libeqat_b200.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
SOURCES = ("api.cu", "attention.cu", "cache.cu", "elementwise.cu", "gemm.cu", "gemv.cu", "noalloc.cu", "prompt.cu", "slim.cu",
           "stream.cu", "wide.cu")


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found (set NVCC or put it on PATH)")


def _older(built, sources) -> bool:
    return not os.path.exists(built) or any(os.path.getmtime(d) > os.path.getmtime(built) for d in sources)


HEADER = os.path.join(ROOT, "include", "eqat.h")


def _stale() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [HEADER])


def marshal_tag() -> str:
    """What the marshalling module fits: this Python and the installed torch.  The module holds it."""
    return f"built for {sys.implementation.cache_tag}, torch {importlib.metadata.version('torch')}."


def marshal_fits(path=None) -> bool:
    with open(path or MARSHAL, "rb") as f:
        return marshal_tag().encode() in f.read()


def _marshal_stale() -> bool:
    return _older(MARSHAL, [os.path.join(CSRC, "marshal.cpp"), HEADER]) or not marshal_fits()


def _build_marshal() -> None:
    """csrc/marshal.cpp against the installed torch (its headers and libraries; nothing of it is built)."""
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    include = [os.path.join(ROOT, "include"), os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += ["-I" + d for d in include] + [f'-DEQAT_BUILT_FOR="{marshal_tag()}"']
    cmd += [os.path.join(CSRC, "marshal.cpp"), "-o", MARSHAL, "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libeqat_b200.so and csrc/marshal.cpp into _marshal.so next to this file; returns the
    library's path."""
    if not force and not _stale():
        if _marshal_stale():
            _build_marshal()
        return LIB
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "--threads", "0",
           "-shared", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
        print(" ".join(cmd))
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)
    _build_marshal()
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
