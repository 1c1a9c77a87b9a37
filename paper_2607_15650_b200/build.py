"""Build libditango.so (sm_100a only) in-tree with nvcc.

    python -m paper_2607_15650_b200.build [--force] [--verbose]

nvcc cross-compiles without a GPU.  The library links the static CUDA runtime and resolves the
one driver entry point it needs (tensor-map encoding) at run time, so it has no link-time
dependency on libcuda.  The Python entry points of the context-free operators are a module of
their own, which needs a C and C++ compiler and Python's and torch's headers (with CUDA); without one of them the library is built
alone.  It is built for one torch, and anew when that is another.
"""
from __future__ import annotations

import importlib.util
import os
import re
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
OPS_LIBS = ("torch_python", "torch_cpu", "c10_cuda", "c10")       # of torch
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def _stale(lib=LIB, files=SOURCES + HEADERS) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in files)


def _torch():
    """(torch's folder, its whole version), without importing it; (None, None) where there is none."""
    spec = importlib.util.find_spec("torch")
    for folder in (spec.submodule_search_locations or [] if spec else []):
        at = os.path.join(folder, "version.py")
        if os.path.exists(at):
            with open(at) as f:
                found = re.search(r"^__version__\s*=\s*['\"]([^'\"]+)", f.read(), re.M)
            if found:
                return folder, found[1]
    return None, None


def _built_for():
    """The version of torch that the module of Python entry points is built for, as left beside it; None where there is none."""
    try:
        with open(OPS_LIB + ".torch") as f:
            return f.read()
    except OSError:
        return None


def _build_ops(force: bool) -> None:
    torch, version = _torch()
    if not force and _built_for() == version and not _stale(OPS_LIB, [OPS_SOURCE, OPS_TENSOR, "ops_tensor.h", HEADERS[-1]]):
        return
    cc, include = shlex.split(os.environ.get("CC") or "gcc"), sysconfig.get_paths()["include"]
    cuda = os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")
    missing = [] if shutil.which(cc[0]) else [cc[0]]
    needed = [os.path.join(include, "Python.h")]
    if torch is None:
        missing.append("torch")
    else:
        needed += [os.path.join(torch, "include", *f.split("/")) for f in ("torch/csrc/autograd/python_variable.h", "c10/cuda/CUDAStream.h")]
        needed += [os.path.join(torch, "lib", f"lib{n}.so") for n in OPS_LIBS] + [os.path.join(cuda, "cuda_runtime_api.h")]
    missing += [f for f in needed if not os.path.exists(f)]
    if missing:
        warnings.warn(f"no Python entry points of the context-free operators: {', '.join(missing)} missing")
        return
    tmp = OPS_LIB + f".tmp{os.getpid()}"
    subprocess.run([*cc, "-O2", "-shared", "-fPIC", "-Wall", "-I" + include, "-I" + os.path.join(torch, "include"), "-I" + cuda,
                    f'-DBUILT_FOR_TORCH="{version}"', "-o", tmp, os.path.join(CSRC, OPS_SOURCE), os.path.join(CSRC, OPS_TENSOR),
                    "-L" + os.path.join(torch, "lib"), *("-l" + n for n in OPS_LIBS), "-lstdc++"], check=True)
    os.replace(tmp, OPS_LIB)
    with open(tmp, "w") as f:
        f.write(version)
    os.replace(tmp, OPS_LIB + ".torch")


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
