"""Builds libetr.so (sm_100a only) with nvcc, and the argument marshalling of the row operators, _args.so, with g++, in-tree,
next to this file."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libetr.so")
SOURCES = ["api.cu", "affinity.cu", "select.cu", "permute.cu", "gate.cu", "gemm_simt.cu", "gemm_tcgen05.cu",
           "gemm_tf32x3.cu",
           "score_tcgen05.cu", "sort.cu", "norm.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared"]


ARGS = os.path.join(HERE, "_args.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "etr.h")


def _stale(target, deps):
    return not os.path.exists(target) or any(os.path.getmtime(p) > os.path.getmtime(target) for p in deps)


def _deps():
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "args.cpp"] + [HEADER]


def build_args(force: bool = False) -> str:
    src = os.path.join(CSRC, "args.cpp")
    if force or _stale(ARGS, [src, HEADER]):
        import torch
        t = os.path.dirname(torch.__file__)
        cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                               *[f"-I{p}" for p in (sysconfig.get_paths()["include"], f"{t}/include", f"{t}/include/torch/csrc/api/include",
                                                    f"{cuda}/include")],
                               "-o", ARGS, src, f"-L{t}/lib", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    return ARGS


def build(force: bool = False, verbose: bool = False) -> str:
    build_args(force)
    if force or _stale(LIB, _deps()):
        nvcc = os.environ.get("NVCC", "nvcc")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + \
              [os.path.join(CSRC, s) for s in SOURCES]
        subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
