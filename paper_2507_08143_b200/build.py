"""Builds the C-ABI library `libcompactor.so` in-tree with nvcc for sm_100a, and beside it `_fastcall.so`, the compiled
argument checks of the entry points that a decoding loop calls per layer and token (host code against torch's headers)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcompactor.so")
SOURCES = ["api.cu", "tensormap.cu", "sweep.cu", "gram.cu", "factor.cu", "score.cu", "select.cu", "compact.cu", "attention.cu", "nll.cu",
           "paged.cu", "decode.cu"]


FASTCALL = os.path.join(HERE, "_fastcall.so")


def _build_fastcall() -> None:
    import sysconfig

    import torch
    root = os.path.join(os.path.dirname(torch.__file__))
    include = [os.path.join(ROOT, "include")]
    system = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
              os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [x for i in include for x in ("-I", i)] + [x for i in system for x in ("-isystem", i)]
    cmd += ["-o", FASTCALL, os.path.join(CSRC, "fastcall.cpp"), "-L", os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu",
            "-ltorch_python"]
    subprocess.run(cmd, check=True)


def _stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(FASTCALL):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(FASTCALL))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "compactor.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; returns its path."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-shared", "-Xcompiler", "-fPIC", "-O3", "-std=c++17", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.run(cmd, check=True)
    _build_fastcall()
    return LIB


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
