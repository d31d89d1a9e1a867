"""Build the HIP plan-search library for gfx950 in-tree.

    python -m paper_2606_16907_amd.build

Compiles every csrc/*.hip file with hipcc, several at a time, and links them into
libtangram_hip.so next to this file.  Floating-point contraction is off (results must match an op-by-op
binary64 evaluation) and packed-FP32 instructions are disabled.
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libtangram_hip.so")
ARCH = os.environ.get("TG_OFFLOAD_ARCH", "gfx950")

FLAGS = ["--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall"]


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))


def build(verbose=False):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)

    with tempfile.TemporaryDirectory() as place, concurrent.futures.ThreadPoolExecutor(os.cpu_count() or 1) as pool:
        objects = [os.path.join(place, os.path.basename(s) + ".o") for s in sources()]
        compiled = [pool.submit(run, [hipcc] + FLAGS + ["-I", os.path.join(ROOT, "include"), "-c", "-o", o, s])
                    for s, o in zip(sources(), objects)]
        for c in compiled:
            c.result()
        tmp = LIB + ".tmp"
        run([hipcc, "--offload-arch=" + ARCH, "-fPIC", "-shared", "-o", tmp] + objects)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)
