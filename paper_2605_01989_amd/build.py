"""Builds libdblp_agg.so (HIP kernels + C-ABI) for gfx950, in-tree: the receiver (dblp_agg.hip) and the worker's
operators (worker_rows.hip, worker_logits.hip; layer_products.hip, layer_update.hip)."""
from __future__ import annotations

import os
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(_HERE, "csrc", f) for f in ("dblp_agg.hip", "worker_rows.hip", "worker_logits.hip", "layer_products.hip", "layer_update.hip")]
LIB = os.path.join(_HERE, "libdblp_agg.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(verbose: bool = False) -> str:
    """Each source by a compiler of its own, then one library of them."""
    with tempfile.TemporaryDirectory() as to:
        objects = [os.path.join(to, os.path.basename(s) + ".o") for s in SRCS]
        compilers = []
        for source, obj in zip(SRCS, objects):
            cmd = [HIPCC, *FLAGS, "-c", "-o", obj, source]
            if verbose:
                print(" ".join(cmd))
            compilers.append((subprocess.Popen(cmd), cmd))
        failed = [cmd for p, cmd in compilers if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.check_call([HIPCC, *FLAGS, "-shared", "-o", LIB, *objects])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
