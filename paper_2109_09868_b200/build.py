"""Builds ``libapproxifer.so`` (sm_100a) in-tree with nvcc, and ``_hosted.so`` (the hosted-model operators' Python binding) with g++.

    python -m paper_2109_09868_b200.build [--force] [--verbose]

Objects go to ``paper_2109_09868_b200/_build/``; the shared libraries are written
next to this file.  nvcc cross-compiles, so no GPU is needed to build.  The two are
built apart: what does not call the hosted-model operators does without the second.
"""
from __future__ import annotations

import argparse
import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OBJDIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libapproxifer.so")
BINDING = os.path.join(HERE, "_hosted.so")  # the hosted-model operators' Python binding (hosted_binding.cpp)

SOURCES = ["api.cu", "tables.cpp", "encode.cu", "decode.cu", "decode_small.cu", "decode_pack.cu", "decode_staged.cu", "locate.cu", "locate_rows.cu", "locate_rows_n8.cu", "locate_rows_n16.cu", "locate_rows_n24.cu", "locate_rows_n32.cu", "host_api.cu", "no_alloc.cu", "hosted_api.cu", "tensor_map.cu", "linear.cu", "linear_tile.cu", "linear_pair.cu", "linear_few.cu", "norm_rope.cu", "attention.cu", "attention_token.cu", "attention_tile.cu", "block_norm.cu", "mx_array.cu", "mx_linear.cu", "mx_pair.cu", "prefix.cu"]
ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]
CFLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall", "--expt-relaxed-constexpr"]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the library cannot be built")
    return exe


MIN_CUDA = (12, 8)  # sm_100a needs CUDA 12.8; kernel parameter blocks above 4 KB (the weight tables) need 12.1


def check_toolkit() -> None:
    """Fails with a clear message when nvcc is older than the kernels need."""
    import re

    out = subprocess.run([nvcc(), "--version"], capture_output=True, text=True).stdout
    m = re.search(r"release (\d+)\.(\d+)", out)
    if m and (int(m.group(1)), int(m.group(2))) < MIN_CUDA:
        raise RuntimeError("nvcc %s.%s is too old: the library needs CUDA %d.%d or later (sm_100a target, kernel "
                           "parameter blocks of up to 32 KB)" % (m.group(1), m.group(2), *MIN_CUDA))


def _stale(target: str, sources) -> bool:
    paths = [os.path.join(CSRC, f) for f in sources] + [os.path.join(INCLUDE, "approxifer.h"), __file__]
    return not os.path.exists(target) or os.path.getmtime(target) < max(os.path.getmtime(p) for p in paths)


def library_is_stale() -> bool:
    return _stale(LIB, [f for f in os.listdir(CSRC) if f != "hosted_binding.cpp"])


def binding_is_stale() -> bool:
    return _stale(BINDING, ["hosted_binding.cpp"])


def is_stale() -> bool:
    return library_is_stale() or binding_is_stale()


def build_binding(verbose: bool = False) -> str:
    """Compiles hosted_binding.cpp against the installed torch's headers (host code only)."""
    import sysconfig

    import torch

    root = os.path.join(os.path.dirname(torch.__file__), "include")
    tmp = BINDING + ".tmp.%d" % os.getpid()
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-isystem", root, "-isystem", os.path.join(root, "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"], "-isystem", cuda,
           os.path.join(CSRC, "hosted_binding.cpp"), "-o", tmp, "-L", os.path.join(os.path.dirname(root), "lib"),
           "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]  # (all loaded by then: importing torch comes first)
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on hosted_binding.cpp:\n%s\n%s" % (r.stdout, r.stderr))
    os.replace(tmp, BINDING)
    return BINDING


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJDIR, os.path.splitext(src)[0] + ".o")
    cmd = [nvcc(), *ARCH, *CFLAGS, "-I", INCLUDE, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("nvcc failed on %s:\n%s\n%s" % (src, r.stdout, r.stderr))
    if verbose:
        print(r.stderr, flush=True)
    return obj


def build_library(verbose: bool = False) -> str:
    check_toolkit()
    os.makedirs(OBJDIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc(), *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    return LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """Both, where they are older than their sources."""
    with concurrent.futures.ThreadPoolExecutor(max_workers=1) as ex:
        binding = ex.submit(build_binding, verbose) if force or binding_is_stale() else None
        if force or library_is_stale():
            build_library(verbose)
        if binding:
            binding.result()
    return LIB


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--force", action="store_true")
    ap.add_argument("--verbose", action="store_true")
    args = ap.parse_args()
    print(build(args.force, args.verbose))
    sys.exit(0)
