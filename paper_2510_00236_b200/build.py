"""Builds the C-ABI library ``csrc/libpestats.so`` in-tree with nvcc for sm_100a.

Run as ``python -m paper_2510_00236_b200.build`` (add ``--force`` to rebuild, ``--verbose`` for the
ptxas resource report).  nvcc cross-compiles, so no GPU is needed to build.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc")
LIB = os.path.join(CSRC, "libpestats.so")
_COMMON = ["pe_host.cuh", "pe_sm100.cuh", "../../include/pestats.h"]
# each source and the headers it includes
SOURCES = {
    "pe_api.cu": _COMMON + ["pe_layout.cuh", "pe_optim.cuh", "pe_stage.cuh", "pe_short.cuh", "pe_simt.cuh", "pe_tc.cuh", "pe_tok.cuh"],
    "pe_muon.cu": _COMMON + ["pe_muon.cuh"],
    "pe_norm.cu": _COMMON + ["pe_norm.cuh"],
}


def _stale(target: str, files) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in files)


def _object(source: str) -> str:
    return os.path.join(CSRC, source.replace(".cu", ".o"))


def _replacing(cmd, target):
    """Runs cmd with its output in a file of its own that then takes the target's place."""
    tmp = target + f".tmp{os.getpid()}"
    subprocess.check_call(cmd + ["-o", tmp])
    os.replace(tmp, target)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not any(_stale(LIB, [source] + headers) for source, headers in SOURCES.items()):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]

    def compile_one(source):
        if force or _stale(_object(source), [source] + SOURCES[source]):
            _replacing(flags + (["-Xptxas", "-v"] if verbose else []) + ["-c", os.path.join(CSRC, source)], _object(source))

    with ThreadPoolExecutor() as pool:
        list(pool.map(compile_one, SOURCES))
    _replacing(flags + ["-shared"] + [_object(source) for source in SOURCES], LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
