"""Builds libmeft.so (HIP, gfx950) in-tree with hipcc.  `python -m paper_2406_04984_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmeft.so")
# the first one's kernels come first in the library
SOURCES = [os.path.join(CSRC, n) for n in ("meft_api.hip", "block_api.hip")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]


def _start(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(procs, verbose):
    failed = False
    for proc in procs:
        text, _ = proc.communicate()
        # the host pass does not know the packed-fp32 target feature and says so once per file: harmless
        out = "\n".join(l for l in text.splitlines() if "packed-fp32-ops" not in l)
        if out.strip() and (verbose or proc.returncode):
            print(out, flush=True)
        failed |= proc.returncode != 0
    if failed:
        raise RuntimeError("hipcc failed")


def build_library(verbose: bool = True) -> str:
    """Compiles the sources side by side and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objects = {s: os.path.splitext(s)[0] + ".o" for s in SOURCES}
    _finish([_start([hipcc, *FLAGS, "-c", "-o", o, s], verbose) for s, o in objects.items()], verbose)
    _finish([_start([hipcc, *FLAGS, "-shared", "-o", LIB, *objects.values()], verbose)], verbose)
    return LIB


if __name__ == "__main__":
    build_library()
    sys.exit(0)
