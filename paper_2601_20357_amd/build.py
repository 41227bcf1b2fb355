"""Builds libtabed.so (HIP, gfx950) in-tree with hipcc.  No GPU is needed to compile."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtabed.so")
SOURCES = ["api.hip", "lmhead.hip", "vocab.hip", "body.hip", "body_gang.hip", "norm_q8.hip", "linear_q8.hip", "cache_q8.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"      # the host pass does not know the device feature
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)


def build_library(verbose: bool = False) -> str:
    """Every source by a compiler of its own, up to eight at a time (160 s one after the other, a minute so), then the link."""
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as pool:
            list(pool.map(lambda so: _run(["hipcc", *FLAGS, "-c", "-o", so[1], os.path.join(CSRC, so[0])], verbose), zip(SOURCES, objects)))
        _run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objects], verbose)
    return LIB


MICRO_SRC = os.path.join(HERE, "microbench", "chip_costs.hip")
MICRO_BIN = os.path.join(HERE, "microbench", "chip_costs")


def build_microbench(verbose: bool = False) -> str:
    """The stand-alone fixed-cost microbenchmark (launch overhead, streaming reads, hand-over variants)."""
    cmd = ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-o", MICRO_BIN, MICRO_SRC]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stderr)
    return MICRO_BIN


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_microbench(verbose=True))
