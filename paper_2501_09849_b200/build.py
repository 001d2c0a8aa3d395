"""Builds libcdl.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and beside it _cdl_calls.so, the compiled part of
the Python binding (argument marshalling, plain C).

Usage: ``python -m paper_2501_09849_b200.build [--force] [--verbose]``.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libcdl.so"
CALLS = PKG / "_cdl_calls.so"

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-DNDEBUG",
    "-shared", "-cudart", "static", "--threads", "0",
]


def sources():
    return sorted(CSRC.glob("*.cu"))


def _stale() -> bool:
    if not LIB.exists() or not CALLS.exists():
        return True
    t = min(LIB.stat().st_mtime, CALLS.stat().st_mtime)
    deps = list(CSRC.glob("*")) + [ROOT / "include" / "cdl.h", Path(__file__)]
    return any(d.stat().st_mtime > t for d in deps)


def _build_calls() -> None:
    tmp = CALLS.with_suffix(f".so.tmp{os.getpid()}")
    subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-std=c11", "-shared", "-fPIC", "-Wall", "-I", sysconfig.get_paths()["include"],
                    "-I", str(ROOT / "include"), "-o", str(tmp), str(CSRC / "cdl_calls.c")], check=True)
    os.replace(tmp, CALLS)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every .cu under csrc/ into libcdl.so and the binding's C file beside it; no-op when up to date."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB.with_suffix(f".so.tmp{os.getpid()}")
    cmd = [nvcc, *NVCC_FLAGS, "-I", str(ROOT / "include"), "-I", str(CSRC)]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += ["-o", str(tmp), *map(str, sources())]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    _build_calls()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
