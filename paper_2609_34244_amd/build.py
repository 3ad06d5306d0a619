"""Build the gfx950 plan-pricing library (libheddle.so) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libheddle.so")
SOURCES = ["profile.cpp", "windows.hip", "price.hip", "search.hip", "evaluate.hip", "distribute.hip", "argmin.hip", "enumerate.hip", "tile.hip",
           "fill.hip", "linear.hip", "gated_ffn.hip", "clip.hip", "norm.hip", "balance.hip", "attention.hip",
           "attention_forward.hip", "attention_backward.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
    # inline asm that names m0, which the compiler keeps for no value of its own here
    "-Wno-inline-asm",
    # no packed fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _hipcc(args, verbose):
    cmd = [HIPCC, *FLAGS, *args]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed ({r.returncode}):\n{err}")
    if err.strip() and verbose:
        print(err, file=sys.stderr)


def build(verbose=False):
    """Compiles the sources, several at a time, and links them."""
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as d, ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        objects = [os.path.join(d, s + ".o") for s in SOURCES]
        list(pool.map(lambda so: _hipcc(["-c", os.path.join(CSRC, so[0]), "-o", so[1]], verbose), zip(SOURCES, objects)))
        _hipcc(["-shared", "-o", tmp, *objects], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
