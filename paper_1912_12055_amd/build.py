"""Compile the HIP library (libnna.so) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libnna.so")
SOURCES = ["nna_plan.hip", "nna_banks.hip", "nna_run.hip", "nna_backward.hip", "nna_kernels.hip", "nna_kernels_fold.hip", "nna_kernels_fft.hip", "nna_kernels_cqf.hip", "nna_kernels_cql.hip", "nna_kernels_short.hip", "nna_kernels_f16.hip", "nna_train.hip", "nna_kernels_split.hip", "nna_kernels_norm.hip", "nna_kernels_decay.hip", "nna_sequence.hip", "nna_kernels_rotate.hip", "nna_kernels_scan.hip", "nna_kernels_adamw.hip", "nna_network.hip"]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=gfx950",
    # packed-FP32 VALU ops are switched off for all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build_library(verbose: bool = False, extra_flags=()) -> str:
    """Always recompiles; returns the path of the shared library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, *HIPCC_FLAGS, *extra_flags, "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
