"""Builds libdit.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _marshal.so (the Python side of its
context-free operators) with the host compiler against torch's headers."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdit.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = [os.path.join(CSRC, "dit_api.cu"), os.path.join(CSRC, "ops_api.cu"), os.path.join(CSRC, "sched.cc")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC"]


def _newest_source_mtime() -> float:
    t = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for name in os.listdir(root):
            t = max(t, os.path.getmtime(os.path.join(root, name)))
    return t


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library if it is missing or older than its sources; returns its path."""
    newest = _newest_source_mtime()
    if not force and all(os.path.exists(p) and os.path.getmtime(p) >= newest for p in (LIB, MARSHAL)):
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + SOURCES
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose:
        print(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    build_marshal()
    return LIB


def build_marshal() -> str:
    """Compiles csrc/marshal.cc against torch and links it to libdit.so (found beside it at run time)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension as X
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    includes = X.include_paths() + [sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}"]
           + [f"-I{d}" for d in includes] + ["-o", MARSHAL, os.path.join(CSRC, "marshal.cc"), f"-L{HERE}", "-l:libdit.so", "-Wl,-rpath,$ORIGIN", f"-L{torch_lib}"]
           + ["-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("the host compiler failed:\n" + res.stdout + res.stderr)
    return MARSHAL


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
