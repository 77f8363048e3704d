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
_COMMON = ["ptx.cuh", "check.cuh", "kv_common.cuh", "kv_attend.cuh", "kv_attend_tile.cuh", "kv_host.cuh", "kv_check.cuh"]
_UNITS = {  # translation units, and the headers that each includes beside the common ones
    "ivf_api.cu": ["scales.cuh", "fused_topk.cuh", "merge.cuh", "prep.cuh", "update.cuh", "pq.cuh", "candidates.cuh", "kv_tables.cuh",
                   "kv_append.cuh", "kv_summary.cuh", "kv_select.cuh", "kv_api.cuh"],
    "kv_whole.cu": ["kv_chunk.cuh", "kv_chunk_tile.cuh", "kv_pages.cuh"],
}
_CHECKED = {"ivf_api.cu"}  # units whose kernels have index checks to switch on


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _deps(unit: str) -> list[str]:
    return [os.path.join(_CSRC, f) for f in [unit, *_UNITS[unit], *_COMMON]] + [os.path.join(_ROOT, "include", "ivf_b200.h")]


def _newer(deps: list[str], path: str) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def _stale(path: str = LIB_PATH) -> bool:
    return any(_newer(_deps(unit), path) for unit in _UNITS)


def _remove(path: str) -> None:
    if os.path.exists(path):
        os.remove(path)


def _write(out: str, cmd) -> None:
    """Runs cmd(file), whose output takes the place of `out` if it comes through."""
    tmp = out + f".{os.getpid()}.tmp"
    try:
        subprocess.check_call(cmd(tmp))
        os.replace(tmp, out)
    finally:
        _remove(tmp)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compiles the units side by side (those whose objects are older than their sources) and links them."""
    out = CHECKED_LIB_PATH if checked else LIB_PATH
    if not force and not _stale(out):
        return out
    folder = os.path.join(_PKG, "build")
    os.makedirs(folder, exist_ok=True)
    cmd = [_nvcc(), "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-Xcompiler", "-fPIC", "-I", os.path.join(_ROOT, "include")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    objects, running, failed = [], [], None
    try:
        for unit in _UNITS:
            other = checked and unit in _CHECKED
            obj = os.path.join(folder, unit.removesuffix(".cu") + ("_checked.o" if other else ".o"))
            objects.append(obj)
            if force or _newer(_deps(unit), obj):
                tmp = obj + f".{os.getpid()}.tmp.o"
                running.append((subprocess.Popen(cmd + (["-DIVF_CHECK_BOUNDS"] if other else []) + ["-c", os.path.join(_CSRC, unit), "-o", tmp]), tmp, obj))
        for process, tmp, obj in running:
            if process.wait() == 0:
                os.replace(tmp, obj)
            else:
                failed = process.args
    finally:  # (one that fails or is broken off leaves nothing behind)
        for process, tmp, _ in running:
            if process.poll() is None:
                process.kill()
                process.wait()
            _remove(tmp)
    if failed:
        raise subprocess.CalledProcessError(1, failed)
    _write(out, lambda tmp: [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", *objects, "-o", tmp])
    return out


def build_bind(force: bool = False) -> str:
    """The CPython module that hands tensors to the block-cache entry points."""
    src, header = os.path.join(_CSRC, "kv_bind.cpp"), os.path.join(_ROOT, "include", "ivf_b200.h")
    if not force and os.path.exists(BIND_PATH) and all(os.path.getmtime(f) <= os.path.getmtime(BIND_PATH) for f in (src, header)):
        return BIND_PATH
    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    libs = os.path.join(base, "lib")
    cmd = lambda tmp: ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-isystem", os.path.join(base, "include"), "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include"), src, "-o", tmp,
           "-L" + libs, "-Wl,-rpath," + libs, "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]
    _write(BIND_PATH, cmd)
    return BIND_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
    print(build_bind(force="--force" in sys.argv))
