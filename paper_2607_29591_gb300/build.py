"""Compile the CUDA library in-tree for sm_103a (nvcc, no cmake).

``build()`` compiles every translation unit of ``csrc/`` in parallel and links
``libreskv.so`` beside this file, and, where torch is installed, ``_bind.so``, the
small calls' way to it from torch tensors (host C++).  Objects go to ``_build/``.
All are git-ignored build products.
"""
from __future__ import annotations

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
BUILD_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libreskv.so")
SOURCES = ["reskv_api.cu", "decode_kernel.cu", "decode_mma.cu", "decode_cluster.cu",
           "construct.cu", "decode_noalloc.cu", "append.cu", "rope.cu", "paged.cu", "paged_attn.cu",
           "paged_attn_blocks.cu", "paged_prefix.cu", "paged_shared.cu", "cross_attn.cu", "cross_general.cu", "cross_blocks.cu", "cross_rows.cu",
           "cross_grad.cu"]
BIND = os.path.join(HERE, "_bind.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I" + INCLUDE,
                "-I" + CSRC]


def nvcc() -> str:
    path = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(path):
        raise RuntimeError("nvcc not found")
    return path


def _deps():
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    return hdrs + [os.path.join(INCLUDE, "reskv.h")]


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD_DIR, src.replace(".cu", ".o"))
    srcp = os.path.join(CSRC, src)
    if _stale(obj, [srcp] + _deps()):
        cmd = [nvcc()] + FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", srcp, "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{res.stderr}")
        if verbose:
            print(res.stderr)
    return obj


def _bind(force: bool) -> None:
    src = os.path.join(CSRC, "bind.cpp")
    spec = importlib.util.find_spec("torch")
    if spec is None:            # the C library by itself needs none
        return
    torch = spec.submodule_search_locations[0]
    if not force and not _stale(BIND, [src, os.path.join(INCLUDE, "reskv.h"), os.path.join(torch, "version.py")]):
        return
    lib = os.path.join(torch, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + INCLUDE, "-I" + os.path.join(torch, "include"),
           "-I" + os.path.join(torch, "include", "torch", "csrc", "api", "include"),
           "-I" + sysconfig.get_paths()["include"], src, "-o", BIND + ".new", "-L" + lib, "-ltorch_python",
           "-ltorch_cpu", "-lc10", "-Wl,-rpath," + lib]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"g++ failed on bind.cpp:\n{res.stderr}")
    os.replace(BIND + ".new", BIND)


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libreskv.so if any source changed; return its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    if force:
        for f in os.listdir(BUILD_DIR):
            os.remove(os.path.join(BUILD_DIR, f))
    with concurrent.futures.ThreadPoolExecutor(len(SOURCES) + 1) as ex:
        bind = ex.submit(_bind, force)
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
        bind.result()
    if force or _stale(LIB, objs):
        cmd = [nvcc()] + ARCH + ["-shared", "-o", LIB] + objs
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"link failed:\n{res.stderr}")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
