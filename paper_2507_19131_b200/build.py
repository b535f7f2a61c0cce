"""Builds the CUDA library (libmixaq.so, sm_100a) in-tree with nvcc.  No JIT cache, no torch extension:
the product is a plain C-ABI shared object declared in include/mixaq.h."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmixaq.so")

# Every binary32 operation must round exactly once and in the written order: no contraction into FMAs
# (explicit fmaf only), IEEE division and square root, no flush-to-zero.
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "--fmad=false", "-prec-div=true", "-prec-sqrt=true", "-ftz=false",
              "-Xcompiler", "-fPIC", "-shared"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "mixaq.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else [])
    # the sources are compiled side by side; libcuda is only needed for the tensor-map encoder, which is resolved lazily, so that
    # the build works without a driver
    with tempfile.TemporaryDirectory() as tmp:
        def compile_one(source):
            obj = os.path.join(tmp, os.path.basename(source) + ".o")
            subprocess.check_call([nvcc] + [f for f in flags if f != "-shared"] + ["-c", "-o", obj, source])
            return obj
        with ThreadPoolExecutor(os.cpu_count() or 1) as pool:
            objects = list(pool.map(compile_one, sources()))
        out = os.path.join(tmp, "libmixaq.so")
        subprocess.check_call([nvcc] + NVCC_FLAGS + ["-o", out] + objects + ["-ldl"])
        new = f"{LIB[:-3]}.{os.getpid()}.so"             # in place at once: another process may be loading the library
        shutil.copyfile(out, new)
        os.replace(new, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
