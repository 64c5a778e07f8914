"""Build libaccordion.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = [os.path.join(HERE, "csrc", "accordion.hip")] + [
    os.path.join(HERE, "csrc", "operators", f"{name}.hip") for name in ("operators", "convolution", "scan", "logprob")]
LIB = os.path.join(HERE, "libaccordion.so")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt",
    # no packed fp32 instructions: some of their forms have given wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def build(verbose: bool = True) -> str:
    """Every source becomes an object, side by side; then they are linked."""
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as where, ThreadPoolExecutor(min(len(SRC), os.cpu_count() or 1)) as pool:
        objects = [os.path.join(where, os.path.splitext(os.path.basename(s))[0] + ".o") for s in SRC]
        list(pool.map(run, [[hipcc()] + FLAGS + ["-c", "-o", o, s] for o, s in zip(objects, SRC)]))
        run([hipcc()] + FLAGS + ["-shared", "-o", LIB] + objects)
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
