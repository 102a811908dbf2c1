"""Builds libdit.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _marshal.so (the Python side of its
context-free operators) with the host compiler against torch's headers."""
from __future__ import annotations

import os
import subprocess
import time

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdit.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = [os.path.join(CSRC, name) for name in ("dit_api.cu", "ops_api.cu", "fp4_api.cu", "prompt_api.cu", "sched.cc")]
OBJECTS = os.path.join(HERE, "_obj")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]


def _newest_source_mtime() -> float:
    t = os.path.getmtime(__file__)                 # (it holds the flags)
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for name in os.listdir(root):
            t = max(t, os.path.getmtime(os.path.join(root, name)))
    return t


def _fresh(obj: str, made_by: str) -> bool:
    """Whether an object was made by this compiler and command, to the end, from the files that its dependency list names as they are now."""
    try:
        named = open(obj + ".d").read().replace("\\\n", " ").split(" : ", 1)[1].split()        # "object : source header ..."
        return open(obj + ".by").read() == made_by and all(os.path.getmtime(p) < os.path.getmtime(obj) for p in named)
    except (OSError, IndexError):
        return False


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library if it is missing or older than its sources; returns its path."""
    newest = _newest_source_mtime()
    if not force and all(os.path.exists(p) and os.path.getmtime(p) >= newest for p in (LIB, MARSHAL)):
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    version = subprocess.run([nvcc, "--version"], capture_output=True, text=True).stdout
    os.makedirs(OBJECTS, exist_ok=True)
    objects = [os.path.join(OBJECTS, os.path.basename(src) + ".o") for src in SOURCES]
    jobs = []                                      # sources are compiled side by side, those whose object is older than what it was made of
    for src, obj in zip(SOURCES, objects):
        cmd = [nvcc] + NVCC_FLAGS + ["-MMD", "-MF", obj + ".d", "-c", src, "-o", obj]
        made_by = "\n".join(cmd + [version])
        if force or not _fresh(obj, made_by):
            if os.path.exists(obj + ".by"):
                os.remove(obj + ".by")
            start = time.time()
            jobs.append((src, obj, made_by, start, subprocess.Popen(cmd[:-4] + (["-Xptxas", "-v"] if verbose else []) + cmd[-4:], stdout=subprocess.PIPE,
                                                                    stderr=subprocess.STDOUT, text=True)))
    done = []
    for src, obj, made_by, start, job in jobs:
        done.append((src, job.communicate()[0], job.returncode))
        if job.returncode == 0:
            os.utime(obj, (start, start))          # (a file that changed meanwhile is newer)
            with open(obj + ".by", "w") as f:
                f.write(made_by)
    if verbose:
        print("".join(out for _, out, _ in done))
    for src, out, code in done:
        if code != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{out}")
    res = subprocess.run([nvcc] + NVCC_FLAGS[:2] + ["-shared", "-o", LIB] + objects, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("linking failed:\n" + res.stdout + res.stderr)
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
