"""Compile the CUDA library in-tree for sm_100a with nvcc, and the functions that call it with torch tensors (no GPU needed to build)."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libflashmesh.so")
SRC = [os.path.join(HERE, "csrc", f) for f in ("flashmesh.cu", "fm_ops.cu")]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared", "--threads", "2"]

# the functions for torch tensors: a Python module beside the library, which it loads from there
HOST = os.path.join(HERE, "_trees.so")
HOST_SRC = os.path.join(HERE, "csrc", "trees_host.cpp")


def _host_command():
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], cuda]
    libs = os.path.join(torch, "lib")
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared"] + ["-I" + d for d in include] + ["-o", HOST, HOST_SRC, "-L" + HERE, "-l:libflashmesh.so", "-L" + libs,
            "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"])


def _run(cmd, what):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(what)
    return res


def _newer(target, sources):
    return os.path.exists(target) and all(os.path.getmtime(s) <= os.path.getmtime(target) for s in sources)


def _sources():
    out = [os.path.join(HERE, "..", "include", "flashmesh.h")]
    for f in os.listdir(os.path.join(HERE, "csrc")):
        if f != os.path.basename(HOST_SRC):
            out.append(os.path.join(HERE, "csrc", f))
    return out


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libflashmesh.so and _trees.so if they are missing or older than a source file; return the library's path."""
    if force or not _newer(LIB, _sources()):
        nvcc = os.environ.get("NVCC", "nvcc")
        res = _run([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + SRC, "nvcc failed building libflashmesh.so")
        if verbose:
            sys.stderr.write(res.stderr)
    if force or not _newer(HOST, [HOST_SRC, _sources()[0]]):
        _run(_host_command(), "g++ failed building _trees.so")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
