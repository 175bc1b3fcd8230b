"""Builds the CUDA library (nvcc, sm_100a; cross-compiles without a GPU) and the Python marshalling module (g++) in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
from typing import List

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libleanstream.so")
SOURCES = ["leanstream.cu", "decoder_ops.cu", "kv4_ops.cu", "kv4_attend_bf16.cu", "kv4_attend_fp16.cu"]
HEADERS = ["ls_common.cuh", "ls_topk.cuh", "ls_kernels.cuh", "ls_cache.cuh", "ls_token.cuh", "ls_hash.cuh",
           "ls_host.cuh", "ls_append.cuh", "ls_attend.cuh", "ls_attend_tile.cuh", "ls_tmem.cuh", "ls_norm.cuh", "ls_kv4.cuh",
           "ls_kv4_attend.cuh", "ls_kv4_shapes.cuh"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC", "--threads", "0",
]


MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")
MARSHAL_PATH = os.path.join(PKG_DIR, "ls_marshal" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: cannot build libleanstream.so")
    return exe


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps: List[str] = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    deps.append(os.path.join(ROOT, "include", "leanstream.h"))
    return any(os.path.exists(p) and os.path.getmtime(p) > t for p in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile ``libleanstream.so`` next to this file when missing or older than its sources."""
    if not force and not _stale():
        return LIB_PATH
    cmd = [_nvcc(), *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-o", LIB_PATH] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)
    return LIB_PATH


def build_marshal(force: bool = False) -> str:
    """Compile the marshalling module next to this file when missing or older than its sources."""
    deps = [MARSHAL_SOURCE, os.path.join(ROOT, "include", "leanstream.h")]
    if not force and os.path.exists(MARSHAL_PATH) and all(os.path.getmtime(p) <= os.path.getmtime(MARSHAL_PATH) for p in deps if os.path.exists(p)):
        return MARSHAL_PATH
    import torch
    from torch.utils.cpp_extension import include_paths

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", sysconfig.get_path("include"),
           "-I", cuda]
    for p in include_paths():
        cmd += ["-isystem", p]
    cmd += [MARSHAL_SOURCE, "-o", MARSHAL_PATH, "-L", lib, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    return MARSHAL_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
