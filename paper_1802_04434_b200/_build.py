"""Compile the CUDA library in-tree with nvcc for sm_100a."""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
SOURCES = [os.path.join(_HERE, "csrc", n) for n in ("signsgd.cu", "variants.cu", "stats.cu", "exchange.cu", "vote_staged.cu",
                                                     "tensors.cu", "fp4_quantise.cu", "fp4_matmul.cu",
                                                     "cross_entropy.cu", "orthogonal.cu")]
HEADERS = [os.path.join(ROOT, "include", "signsgd.h")] + [
    os.path.join(_HERE, "csrc", n) for n in ("device_common.cuh", "host_common.h", "vote_launch.h", "step_rows.cuh", "host_calls.h", "dtypes.cuh", "fp4.cuh", "sm100.cuh",
                                     "tensor_map.h", "half_product.cuh")]
LIB = os.path.join(_HERE, "libsignsgd_b200.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-lineinfo", "-std=c++17",
    "--fmad=false",            # no silent contraction: fused operations are written explicitly
    "-Xcompiler", "-fPIC", "-shared",
    "-I", os.path.join(ROOT, "include"),
]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return exe


def is_fresh() -> bool:
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(p) <= t for p in SOURCES + HEADERS + [os.path.abspath(__file__)])


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libsignsgd_b200.so next to this file; returns its path."""
    if not force and is_fresh():
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    compile_flags = [f for f in NVCC_FLAGS if f != "-shared"] + (["-Xptxas", "-v"] if verbose else [])

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
        if verbose:
            print(res.stdout + res.stderr)

    # a compiler for each source, side by side: two minutes one after the other
    with tempfile.TemporaryDirectory() as objects, concurrent.futures.ThreadPoolExecutor(os.cpu_count()) as pool:
        outs = [os.path.join(objects, os.path.basename(s) + ".o") for s in SOURCES]
        list(pool.map(lambda pair: run([nvcc(), *compile_flags, "-c", "-o", *pair]), zip(outs, SOURCES)))
        run([nvcc(), *NVCC_FLAGS, "-o", tmp, *outs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
