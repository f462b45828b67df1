"""Builds the CUDA library in-tree: csrc/*.cu -> libgrouter.so (sm_100a only); with debug=True the checked build
libgrouter_debug.so, whose kernels test data-derived indices before use (grouter_checked_build in the header)."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libgrouter.so")
LIB_DEBUG = os.path.join(PKG, "libgrouter_debug.so")
SOURCES = ["api.cu", "plan.cu", "permute.cu", "gemm.cu", "route.cu", "stats.cu", "ep.cu", "norm.cu", "balance.cu", "linear.cu", "linear_small.cu", "adamw.cu",
           "quant.cu", "rmsnorm.cu", "gated.cu", "fp8_gemm.cu", "fp8_small.cu"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "grouter.h")]
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compiles if the library is missing or older than any source.  Returns its path."""
    lib = LIB_DEBUG if debug else LIB
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= _newest_source_mtime():
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = f"{lib}.{os.getpid()}.tmp"      # several processes may build at once: each writes its own file, then renames it
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-shared", "-t", "0",
           "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", tmp]
    if debug:
        cmd += ["-DGROUTER_DEBUG_BOUNDS"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError(f"nvcc failed building {os.path.basename(lib)}")
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
