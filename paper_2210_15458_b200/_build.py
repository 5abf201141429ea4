"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libarith_sampling.so")
# the same sources with computed indices checked (-DAS_BOUNDS_CHECK, as_bounds.cuh): for the tests
LIB_CHECKED = os.path.join(_HERE, "libarith_sampling_check.so")
SOURCES = ["as_api.cu", "as_edit.cu", "as_cache4.cu", "as_pages.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _newest_source_mtime() -> float:
    m = 0.0
    for d in (CSRC, os.path.join(os.path.dirname(_HERE), "include")):
        for f in os.listdir(d):
            if f.endswith((".cu", ".cuh", ".h")):
                m = max(m, os.path.getmtime(os.path.join(d, f)))
    return m


def _depends(path: str, seen=None) -> set:
    """A source file and the project headers that it includes, directly or not."""
    seen = set() if seen is None else seen
    path = os.path.normpath(path)
    if path not in seen and os.path.exists(path):
        seen.add(path)
        with open(path) as f:
            for name in re.findall(r'^\s*#include "([^"]+)"', f.read(), re.M):
                _depends(os.path.join(os.path.dirname(path), name), seen)
    return seen


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile csrc/*.cu into libarith_sampling.so (checked: libarith_sampling_check.so, with
    -DAS_BOUNDS_CHECK) if it is missing or stale: the sources whose object file is older than what
    they include, side by side, then one link."""
    lib = LIB_CHECKED if checked else LIB
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= _newest_source_mtime():
        return lib
    objdir = os.path.join(_HERE, "_build_check" if checked else "_build_lib")
    os.makedirs(objdir, exist_ok=True)
    flags = NVCC_FLAGS + (["-DAS_BOUNDS_CHECK"] if checked else []) + (["-Xptxas", "-v"] if verbose else [])

    def compile_one(name):
        src, obj = os.path.join(CSRC, name), os.path.join(objdir, name[:-3] + ".o")
        newest = max(os.path.getmtime(f) for f in _depends(src))
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < newest:
            part = obj + ".tmp.%d" % os.getpid()
            subprocess.check_call([_nvcc()] + flags + ["-c", "-o", part, src])
            os.replace(part, obj)
        return obj

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    tmp = lib + ".tmp.%d" % os.getpid()
    subprocess.check_call([_nvcc()] + NVCC_FLAGS + ["-shared", "-o", tmp] + objs)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
