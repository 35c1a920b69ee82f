"""Compile libmpt.so in place for gfx950 with hipcc (no torch involved)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
SRCS = [os.path.join(CSRC, f) for f in ("mpt.hip", "ctx.hip", "greedy.hip", "layout.hip", "pinned.hip")]
KV_SRCS = [os.path.join(CSRC, f) for f in ("attention_wide.hip", "attention_narrow.hip", "attention.hip", "kv.hip")]
LIB = os.path.join(PKG, "libmpt.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

COMMON = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 instructions anywhere
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]
# the solver's only floating point is exact integer keys held as doubles:
# finite by construction, so min needs no NaN quieting. The cache's sources
# are built without it: their NaNs are the caller's.
SOLVER = ["-fno-honor-nans"]


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as d:
        jobs, objects = [], []
        for srcs, flags in ((KV_SRCS, []), (SRCS, SOLVER)):
            for src in srcs:
                obj = os.path.join(d, os.path.basename(src) + ".o")
                objects.append(obj)
                jobs.append([HIPCC, *COMMON, *flags, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj])
        link = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", tmp,
                "-L", "/opt/rocm/lib", "-lrocprofiler-sdk-roctx", "-Wl,-rpath,/opt/rocm/lib"]
        if verbose:
            print("\n".join(" ".join(c) for c in (*jobs, link)), flush=True)
        with ThreadPoolExecutor(8) as pool:
            list(pool.map(subprocess.check_call, jobs))
        subprocess.check_call(link)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
