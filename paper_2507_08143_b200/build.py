"""Builds the C-ABI library `libcompactor.so` in-tree with nvcc for sm_100a, and beside it `_fastcall`, the compiled
argument checks of the entry points that a decoding loop calls per layer and token (host code against torch's headers)."""
from __future__ import annotations

import os
import re
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcompactor.so")
SOURCES = ["api.cu", "tensormap.cu", "sweep.cu", "gram.cu", "factor.cu", "score.cu", "select.cu", "compact.cu", "attention.cu", "nll.cu",
           "paged.cu", "decode.cu"]
HEADER = os.path.join(ROOT, "include", "compactor.h")
FASTCALL_SOURCE = "fastcall.cpp"


def _stale(path: str, sources) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(s) > os.path.getmtime(path) for s in sources)


def _compile(cmd, out: str) -> None:
    """Runs a compiler into a file beside `out` and moves it there, so that no other process loads half of it."""
    part = f"{out}.{os.getpid()}.part"
    try:
        subprocess.run(cmd + ["-o", part], check=True)
        os.replace(part, out)
    finally:
        if os.path.exists(part):
            os.remove(part)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; returns its path."""
    if not force and not _stale(LIB, [HEADER] + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != FASTCALL_SOURCE]):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-shared", "-Xcompiler", "-fPIC", "-O3", "-std=c++17", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    _compile(cmd, LIB)
    return LIB


def fastcall_path() -> str:
    """Where the compiled checks for this Python and this torch are.  They read tensors through torch's inline accessors, so that a file built
    against others must not be loaded: the name says what it was built against."""
    import torch
    against = re.sub(r"\W+", "_", f"torch{torch.__version__}_abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}")
    return os.path.join(HERE, f"_fastcall.{against}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_fastcall(force: bool = False) -> str:
    """Compile the argument checks if they are missing for this Python and torch or older than their sources; returns their path."""
    out, source = fastcall_path(), os.path.join(CSRC, FASTCALL_SOURCE)
    if not force and not _stale(out, [HEADER, source]):
        return out
    import torch
    root = os.path.dirname(torch.__file__)
    system = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
              os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include")]
    cmd += [x for i in system for x in ("-isystem", i)]
    cmd += [source, "-L", os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    _compile(cmd, out)
    return out


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    build_fastcall(force=True)
    print(LIB)
