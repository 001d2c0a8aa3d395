"""Builds libcdl.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and beside it _cdl_calls, the compiled part of the Python
binding (argument marshalling, plain C), named for the interpreter that it is built with and for.

The library needs nvcc alone.  Without a C compiler or this Python's headers it is built all the same, with a warning: only the
language-model calls from Python need the other.

Usage: ``python -m paper_2501_09849_b200.build [--force] [--verbose]``.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import warnings
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libcdl.so"
CALLS = PKG / ("_cdl_calls" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-DNDEBUG",
    "-shared", "-cudart", "static", "--threads", "0",
]


def sources():
    return sorted(CSRC.glob("*.cu"))


def _stale(target, deps) -> bool:
    return not target.exists() or any(d.stat().st_mtime > target.stat().st_mtime for d in [*deps, Path(__file__)])


def _build_library(verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB.with_suffix(f".so.tmp{os.getpid()}")
    cmd = [nvcc, *NVCC_FLAGS, "-I", str(ROOT / "include"), "-I", str(CSRC)]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += ["-o", str(tmp), *map(str, sources())]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)


def _build_calls() -> None:
    include, cc = Path(sysconfig.get_paths()["include"]), os.environ.get("CC", "gcc")
    missing = "this Python's headers" if not (include / "Python.h").exists() else (f"the C compiler ({cc})" if shutil.which(cc.split()[0]) is None else None)
    if missing:
        warnings.warn(f"{CALLS.name} is not built, {missing} not found: the language-model calls cannot be made from Python (libcdl.so is complete)")
        return
    tmp = CALLS.with_name(f"{CALLS.name}.tmp{os.getpid()}")
    subprocess.run([*cc.split(), "-O2", "-std=c11", "-shared", "-fPIC", "-Wall", "-I", str(include), "-I", str(ROOT / "include"), "-o", str(tmp),
                    str(CSRC / "cdl_calls.c")], check=True)
    os.replace(tmp, CALLS)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every .cu under csrc/ into libcdl.so and the binding's C file beside it; what is up to date stays."""
    header = ROOT / "include" / "cdl.h"
    if force or _stale(LIB, [d for d in CSRC.glob("*") if d.suffix != ".c"] + [header]):
        _build_library(verbose)
    if force or _stale(CALLS, [CSRC / "cdl_calls.c", header]):
        _build_calls()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
