"""Build libditango.so (sm_100a only) in-tree with nvcc.

    python -m paper_2607_15650_b200.build [--force] [--verbose]

nvcc cross-compiles without a GPU.  The library links the static CUDA runtime and resolves the
one driver entry point it needs (tensor-map encoding) at run time, so it has no link-time
dependency on libcuda.  The Python entry points of the context-free operators are a module of
their own, which needs a C and C++ compiler and Python's and torch's headers; without the compiler or Python's headers the library is
built alone.
"""
from __future__ import annotations

import importlib.util
import os
import shlex
import shutil
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libditango.so")
SOURCES = ["api.cu", "attn_states.cu", "state_merge.cu", "plan.cu", "planner.cu", "ops_api.cu", "rope.cu", "add_rmsnorm.cu",
           "cross_attn.cu", "cross_tiles.cu", "adapter_linear.cu", "adapter_tiles.cu", "packed_attn.cu",
           "packed_tiles.cu"]
HEADERS = ["dt_internal.h", "ops.h", "cross_attn.h", "adapter_linear.h", "packed_attn.h", "tile_wait.cuh", "ptx_sm100.cuh", os.path.join("..", "..", "include", "ditango.h")]
# Python entry points of the context-free operators, for this interpreter
OPS_LIB = os.path.join(HERE, "_ditango_ops" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
OPS_SOURCE, OPS_TENSOR = "ops_py.c", "ops_tensor.cpp"      # (the second against torch's headers)
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def _stale(lib=LIB, files=SOURCES + HEADERS) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in files)


def _build_ops(force: bool) -> None:
    if not force and not _stale(OPS_LIB, [OPS_SOURCE, OPS_TENSOR, "ops_tensor.h", HEADERS[-1]]):
        return
    cc, include = shlex.split(os.environ.get("CC") or "gcc"), sysconfig.get_paths()["include"]
    if shutil.which(cc[0]) is None or not os.path.exists(os.path.join(include, "Python.h")):
        warnings.warn(f"no Python entry points of the context-free operators: {cc[0]} or {include}/Python.h is missing")
        return
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    tmp = OPS_LIB + f".tmp{os.getpid()}"
    subprocess.run([*cc, "-O2", "-shared", "-fPIC", "-Wall", "-I" + include, "-I" + os.path.join(torch, "include"),
                    "-I" + os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include"), "-o", tmp, os.path.join(CSRC, OPS_SOURCE),
                    os.path.join(CSRC, OPS_TENSOR), "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-lstdc++"], check=True)
    os.replace(tmp, OPS_LIB)


def _build_lib(force: bool, verbose: bool) -> None:
    if not force and not _stale(LIB):
        return
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", 
           "--threads", "8", "-o", tmp]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, f) for f in SOURCES]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)


def build(force: bool = False, verbose: bool = False) -> str:
    _build_lib(force, verbose)
    _build_ops(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
