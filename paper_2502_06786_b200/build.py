"""Builds the CUDA library in-tree with nvcc for sm_100a, and beside it the small C++ module through which Python makes the
serving calls (g++, torch's headers).  No JIT cache.

    python -m paper_2502_06786_b200.build [--force] [-v] [--library-only]

With --library-only (``build_library(serving=False)``) the module is left out: the C ABI and all other Python calls work without it.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmatq.so")
MODULE = os.path.join(HERE, "_serving.so")
SOURCES = ["api.cu", "quantize.cu", "slice_pack.cu", "gemv.cu", "gemm_multi.cu", "gemm_multi_static.cu",
           "tokens.cu", "gemm_a8.cu", "kv_append.cu", "attn_paged.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "-Wno-deprecated-gpu-targets"]


def _stale(serving: bool = True) -> bool:
    made = [LIB, MODULE] if serving else [LIB]
    if not all(os.path.exists(f) for f in made):
        return True
    t = min(os.path.getmtime(f) for f in made)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "matq.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False, serving: bool = True) -> str:
    if not force and not _stale(serving):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    build_dir = os.path.join(HERE, "_build")
    os.makedirs(build_dir, exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(build_dir, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = [nvcc, *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd[1:1] = ["-Xptxas", "-v"]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if out.strip() and (verbose or p.returncode):
            print(f"--- {src}\n{out}", file=sys.stderr)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.run([nvcc, "-shared", "-o", LIB, *objs, "-cudart", "static"], check=True)
    if serving:
        build_module(nvcc)
    return LIB


def build_module(nvcc: str) -> str:
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(nvcc))
    includes = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
                os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include")]
    for i in includes:
        cmd += ["-isystem", i]
    cmd += [os.path.join(CSRC, "serving_module.cpp"), "-o", MODULE, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda",
            "-L", HERE, "-l:libmatq.so", "-Wl,-rpath,$ORIGIN"]
    subprocess.run(cmd, check=True)
    return MODULE


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv, serving="--library-only" not in sys.argv))
