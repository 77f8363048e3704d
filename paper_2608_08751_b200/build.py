"""Builds the C-ABI library in-tree with nvcc for sm_100a (cross-compiles without a GPU).

Two variants: the regular library, and a checked one (-DIVF_CHECK_BOUNDS) whose kernels verify their
shared-memory, tensor-memory and global indices and report the first violation through the status
word instead of touching memory out of range -- selected at load time with IVF_B200_CHECKED=1.  Beside
them the marshalling module of the block-cache operators (host code only, built with g++)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
_CSRC = os.path.join(_PKG, "csrc")
LIB_PATH = os.path.join(_PKG, "libivf_b200.so")
CHECKED_LIB_PATH = os.path.join(_PKG, "libivf_b200_checked.so")
BIND_PATH = os.path.join(_PKG, "_kv_bind.so")
_SOURCES = ["ivf_api.cu"]
_HEADERS = ["ptx.cuh", "check.cuh", "scales.cuh", "fused_topk.cuh", "merge.cuh", "prep.cuh", "update.cuh", "pq.cuh",
            "candidates.cuh", "kv_common.cuh", "kv_tables.cuh", "kv_append.cuh", "kv_summary.cuh", "kv_select.cuh",
            "kv_attend.cuh", "kv_attend_tile.cuh", "kv_api.cuh"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _stale(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    deps = [os.path.join(_CSRC, f) for f in _SOURCES + _HEADERS] + [os.path.join(_ROOT, "include", "ivf_b200.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    out = CHECKED_LIB_PATH if checked else LIB_PATH
    if not force and not _stale(out):
        return out
    tmp = out + f".{os.getpid()}.tmp"
    cmd = [_nvcc(), "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(_ROOT, "include")]
    if checked:
        cmd += ["-DIVF_CHECK_BOUNDS"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(_CSRC, s) for s in _SOURCES] + ["-o", tmp]
    subprocess.check_call(cmd)
    os.replace(tmp, out)
    return out


def build_bind(force: bool = False) -> str:
    """The CPython module that hands tensors to the block-cache entry points."""
    src, header = os.path.join(_CSRC, "kv_bind.cpp"), os.path.join(_ROOT, "include", "ivf_b200.h")
    if not force and os.path.exists(BIND_PATH) and all(os.path.getmtime(f) <= os.path.getmtime(BIND_PATH) for f in (src, header)):
        return BIND_PATH
    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    tmp = BIND_PATH + f".{os.getpid()}.tmp"
    libs = os.path.join(base, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-isystem", os.path.join(base, "include"), "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include"), src, "-o", tmp,
           "-L" + libs, "-Wl,-rpath," + libs, "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]
    subprocess.check_call(cmd)
    os.replace(tmp, BIND_PATH)
    return BIND_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
    print(build_bind(force="--force" in sys.argv))
