"""Compile the CUDA library in-tree for sm_100a with nvcc, and the functions that call it with torch tensors (no GPU needed to build)."""
from __future__ import annotations

import importlib.metadata
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


def _built_for():
    """What _trees.so is compiled and linked against, as it is written into the module: another torch or Python may have other
    layouts and symbols, whatever the files' times."""
    try:
        torch = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:        # (a source tree on the path)
        torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    return f"fm built for torch {torch}, {sysconfig.get_config_var('SOABI')};"


def _host_command():
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], cuda]
    libs = os.path.join(torch, "lib")
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f'-DFM_BUILT_FOR="{_built_for()}"'] + ["-I" + d for d in include] + ["-o", HOST, HOST_SRC, "-L" + HERE, "-l:libflashmesh.so", "-L" + libs,
            "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"])


def _run(cmd, what):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(what)
    return res


def _newer(target, sources):
    return os.path.exists(target) and all(os.path.getmtime(s) <= os.path.getmtime(target) for s in sources)


def _host_fits():
    """Is _trees.so there, newer than its sources and built for this torch and Python?"""
    if not _newer(HOST, [HOST_SRC, _sources()[0]]):
        return False
    with open(HOST, "rb") as f:
        return _built_for().encode() in f.read()


def _sources():
    out = [os.path.join(HERE, "..", "include", "flashmesh.h")]
    for f in os.listdir(os.path.join(HERE, "csrc")):
        if f != os.path.basename(HOST_SRC):
            out.append(os.path.join(HERE, "csrc", f))
    return out


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libflashmesh.so and _trees.so if they are missing or older than a source file (the latter also if it is for another torch or
    Python); return the library's path."""
    if force or not _newer(LIB, _sources()):
        nvcc = os.environ.get("NVCC", "nvcc")
        res = _run([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + SRC, "nvcc failed building libflashmesh.so")
        if verbose:
            sys.stderr.write(res.stderr)
    if force or not _host_fits():
        _run(_host_command(), "g++ failed building _trees.so")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
