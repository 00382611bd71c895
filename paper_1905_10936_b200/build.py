"""Builds libef.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the native half of ops.py."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libef.so")
DEBUG_LIB = os.path.join(PKG, "libef_debug.so")      # the checked build (-DEF_DEBUG)
SOURCES = [os.path.join(CSRC, n) for n in ("ef_lib.cu", "ef_vote.cu", "ef_topk.cu", "ef_norm.cu",
                                             "ef_checkpoint.cu", "ef_wgrad.cu", "ef_policy.cu")]
DEPS = SOURCES + [os.path.join(CSRC, "ef_kernels.cuh"), os.path.join(CSRC, "ef_internal.h"),
                  os.path.join(CSRC, "ef_rows.cuh"),
                  os.path.join(ROOT, "include", "ef.h")]

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-lineinfo",
    "--threads", "0",                   # sources compile side by side
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-fmad=false",                      # no implicit contraction: every fused op is explicit
    "-Xcompiler", "-fPIC", "-shared",
    "-ldl",                             # NVTX (header-only) looks for an attached tool with dlopen
]


TORCH_BINDING = os.path.join(PKG, "_ef_torch.so")    # native half of ops.py
TORCH_SOURCES = [os.path.join(CSRC, "ef_torch.cpp"), os.path.join(ROOT, "include", "ef.h")]


def nvcc_path() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Builds libef.so, or with debug=True the checked build libef_debug.so (every kernel
    validates its work item against the problem's sizes)."""
    lib = DEBUG_LIB if debug else LIB
    if not force and os.path.exists(lib):
        newest = max(os.path.getmtime(p) for p in DEPS)
        if os.path.getmtime(lib) >= newest:
            return lib
    cmd = ([nvcc_path()] + NVCC_FLAGS + (["-DEF_DEBUG"] if debug else [])
           + (["-Xptxas", "-v"] if verbose else []) + ["-o", lib] + SOURCES)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose:
        sys.stderr.write(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    return lib


def build_torch_binding(force: bool = False) -> str:
    """Builds _ef_torch.so in-tree with g++ against the installed torch, again where that is another one."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    stamp, built_for = TORCH_BINDING + ".stamp", torch.__version__
    if not force and os.path.exists(TORCH_BINDING) and os.path.exists(stamp):
        with open(stamp) as f:
            same = f.read() == built_for
        if same and os.path.getmtime(TORCH_BINDING) >= max(os.path.getmtime(p) for p in TORCH_SOURCES):
            return TORCH_BINDING
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           f'-DEF_TORCH_VERSION="{built_for}"']
    for inc in cpp_extension.include_paths() + [sysconfig.get_paths()["include"], cuda]:
        cmd += ["-isystem", inc]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd += [TORCH_SOURCES[0], "-o", TORCH_BINDING, "-L", libs, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    with open(stamp, "w") as f:
        f.write(built_for)
    return TORCH_BINDING


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
    print(build_torch_binding())
