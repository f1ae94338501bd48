"""Builds libdblp_agg.so (HIP kernels + C-ABI) for gfx950, in-tree: the receiver (dblp_agg.hip) and the worker's
operators (worker_rows.hip, worker_logits.hip; layer_products.hip, layer_update.hip)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(_HERE, "csrc", f) for f in ("dblp_agg.hip", "worker_rows.hip", "worker_logits.hip", "layer_products.hip", "layer_update.hip")]
LIB = os.path.join(_HERE, "libdblp_agg.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-shared", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(verbose: bool = False) -> str:
    cmd = [HIPCC, *FLAGS, "-o", LIB, *SRCS]
    if verbose:
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
