"""Builds libpsa.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and psa_marshal.so, the compiled part of the Python binding, with g++.

    python -m paper_2012_01114_b200.build [--force] [--verbose]

The shared objects land next to this file so that they travel with the source tree.
"""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpsa.so")
MARSHAL = os.path.join(HERE, "psa_marshal.so")
SOURCES = ["psa_api.cu", "psa_f32.cu", "psa_f32_tensor.cu", "psa_f32_attn_tensor.cu", "psa_gemm.cu", "psa_attn.cu", "psa_attn_persist.cu", "psa_attn_wide.cu", "psa_noalloc.cu", "psa_selftest.cu", "psa_pipes.cu", "psa_prompt.cu", "psa_cache_append.cu", "psa_cache_attn.cu", "psa_pages.cu"]


def _sources():
    return [os.path.join(CSRC, s) for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]


def _deps():
    out = _sources()
    out += [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    out.append(os.path.join(os.path.dirname(HERE), "include", "psa.h"))
    return out


def build_marshal(force: bool = False, verbose: bool = False) -> str:
    """psa_marshal.so, against the installed torch (whose libraries are in the process when it is loaded)."""
    source = os.path.join(CSRC, "psa_marshal.cpp")
    newest = max(os.path.getmtime(p) for p in (source, os.path.join(os.path.dirname(HERE), "include", "psa.h")))
    if not force and os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= newest:
        return MARSHAL
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    tmp = MARSHAL + ".%d.tmp" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-DTORCH_EXTENSION_NAME=psa_marshal", "-DTORCH_API_INCLUDE_EXTENSION_H",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    cmd += ["-I" + d for d in (os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], os.path.join(cuda, "include"))]
    cmd += ["-o", tmp, source, "-L" + os.path.join(root, "lib")] + ["-l" + n for n in ("c10", "c10_cuda", "torch_cpu", "torch", "torch_python")]
    if verbose:
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    os.replace(tmp, MARSHAL)
    return MARSHAL


def build_library(force: bool = False, verbose: bool = False) -> str:
    """libpsa.so; needs nvcc and its host compiler only."""
    newest = max(os.path.getmtime(p) for p in _deps())
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= newest:
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".%d.tmp" % os.getpid()
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-Xcompiler", "-fPIC,-O2", "-shared", "-cudart", "static",
           "-o", tmp] + os.environ.get("PSA_NVCC_FLAGS", "").split() + _sources()
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """The library, and behind it the binding's compiled part, which needs torch: without torch there is no Python to call it from, and the library stands alone."""
    lib = build_library(force, verbose)
    if importlib.util.find_spec("torch") is None:
        print("torch is not installed: psa_marshal.so, the compiled part of the Python binding, is not built", file=sys.stderr)
    else:
        build_marshal(force, verbose)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
