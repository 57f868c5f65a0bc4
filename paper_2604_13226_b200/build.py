"""Builds the CUDA library in-tree: ``nvcc`` for sm_100a only, one shared object next to this file; and, in a step of its own, the
Python module that marshals the calls of a decode step (``g++``, PyTorch's and Python's headers), one for each version of both."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libkvp.so")
SOURCES = ["kvp_api.cu", "kvp_kernels.cu", "kvp_attn_sm100.cu", "kvp_attn_pair.cu", "kvp_compose_noalloc.cu",
           "kvp_paged.cu", "kvp_paged_attn.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]


def _stale(path: str, *kinds: str) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(kinds)] + [os.path.join(_HERE, "..", "include", "kvp.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every ``.cu`` under ``csrc/`` into ``libkvp.so`` (skipped when up to date)."""
    if not force and not _stale(LIB_PATH, ".cu", ".cuh", ".h"):
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = os.environ.get("KVP_NVCC_EXTRA", "").split()       # extra compiler flags, for experiments
    objs = []
    for s in SOURCES:
        o = os.path.join(CSRC, s.replace(".cu", ".o"))
        cmd = [nvcc, *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, s), "-o", o]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        subprocess.check_call(cmd)
        objs.append(o)
    tmp = LIB_PATH + f".{os.getpid()}.tmp"
    subprocess.check_call([nvcc, "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


def calls_path() -> str:
    """Where the marshalling module for this Python and this PyTorch lies: it reads tensors as their headers lay them out."""
    import torch
    return os.path.join(_HERE, f"_kvp_calls-torch{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_calls(force: bool = False) -> str:
    """Compile ``kvp_calls.cpp`` against the PyTorch that is installed (skipped when up to date)."""
    path = calls_path()
    if not force and not _stale(path, ".cpp"):
        return path
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    tmp = path + f".{os.getpid()}.tmp"
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-shared", f"-I{torch}/include",
                           f"-I{torch}/include/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}", os.path.join(CSRC, "kvp_calls.cpp"),
                           "-o", tmp, f"-L{torch}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, path)
    return path


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    if importlib.util.find_spec("torch"):
        print(build_calls(force="--force" in sys.argv))
