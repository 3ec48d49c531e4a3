"""Builds the CUDA library in-tree: ``python -m paper_2509_19729_b200.build``.

nvcc cross-compiles for sm_100a without a GPU.  The shared object lands next to this file so that it travels
with the source tree; nothing is installed into site-packages and nothing is JIT-cached elsewhere.
"""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

HERE = Path(__file__).resolve().parent
CSRC = HERE / "csrc"
INCLUDE = HERE.parent / "include"
LIB = HERE / "libamoeba.so"
LIB_CHECKED = HERE / "libamoeba_checked.so"  # the same sources with -DAMOEBA_CHECK_ITEMS: every work item is tested
#                                              against the extent of its buffers before it is moved
SOURCES = ["plan.cpp", "block_tables.cu", "kv_reshard.cu", "weights_reshard.cu", "append_kv.cu", "attend.cu", "attend_many.cu",
           "scores.cu", "evict_kv.cu", "cache_maps.cu"]
HEADERS = ["plan.hpp", "launch.hpp", "copy_engine.cuh", "kv_items.cuh", "w_items.cuh", "cache_view.cuh", "walk.cuh", "attend.cuh",
           "warp_mma.cuh", "umma.cuh", "cache_maps.hpp"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
    "-Xcompiler", "-fvisibility=hidden", "-shared", "-cudart", "static", "--threads", "0",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build(checked: bool = False) -> bool:
    lib = LIB_CHECKED if checked else LIB
    if not lib.exists():
        return True
    t = lib.stat().st_mtime
    deps = [CSRC / s for s in SOURCES + HEADERS] + [INCLUDE / "amoeba.h"]
    return any(d.stat().st_mtime > t for d in deps)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> Path:
    lib = LIB_CHECKED if checked else LIB
    if not force and not needs_build(checked):
        return lib
    tmp = lib.with_suffix(f".tmp{os.getpid()}.so")
    cmd = [_nvcc(), *NVCC_FLAGS, f"-I{INCLUDE}", f"-I{CSRC}"]
    if checked:
        cmd += ["-DAMOEBA_CHECK_ITEMS"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [str(CSRC / s) for s in SOURCES] + ["-o", str(tmp)]
    subprocess.run(cmd, check=True)
    os.replace(tmp, lib)
    return lib


def torch_calls_path() -> Path:
    """The serving operators' Python calls on torch tensors.  The module reads tensors by the C++ layout of the Python and the torch
    that it was built for, so it is named after them: another version builds its own."""
    import torch

    return HERE / f"_torch_calls.{sys.implementation.cache_tag}-torch{torch.__version__}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}.so"


def torch_calls_stale() -> bool:
    lib, deps = torch_calls_path(), [CSRC / "torch_calls.cpp", INCLUDE / "amoeba.h"]
    return not lib.exists() or any(d.stat().st_mtime > lib.stat().st_mtime for d in deps)


def build_torch_calls(force: bool = False) -> Path:
    """The CPython module between torch tensors and the C library.  It binds the library's functions when it is loaded,
    by then in the process, so that the checked build can stand in for the normal one."""
    lib = torch_calls_path()
    if not force and not torch_calls_stale():
        return lib
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths, library_paths

    tmp = lib.with_suffix(f".tmp{os.getpid()}.so")
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-fvisibility=hidden", f"-I{INCLUDE}",
           f"-I{sysconfig.get_path('include')}", *[f"-I{p}" for p in include_paths("cuda")],
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", str(CSRC / "torch_calls.cpp"),
           *[f"-L{p}" for p in library_paths()], "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-o", str(tmp)]
    subprocess.run(cmd, check=True)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
    print(build_torch_calls(force="--force" in sys.argv))
