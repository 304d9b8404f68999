"""Build librkv.so in-tree with hipcc for gfx950.

    python -m paper_2606_15157_amd.build
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librkv.so")
SOURCES = ["attend.hip", "host.cpp", "prefill.hip", "decode.hip", "entropy.hip", "fullspan.hip", "tova.hip", "handoff.hip", "noalloc.hip", "window.hip",
           "paged.cpp", "pages.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Wall", "-Wno-unused-function",
    # keep the compiler from emitting packed fp32 arithmetic
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep single-lane atomics as written: the atomic optimizer turns them into a wave-wide
    # form whose result is read back at once, which would wait for the atomic's round trip
    # where the code only needs the result an iteration later
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return os.path.join(rocm, "bin", "hipcc")


def build(verbose: bool = False) -> str:
    """Compiles every source (side by side: the attention's instances take the longest) and links them."""
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        noise = "is not a recognized feature for this target"
        err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)

    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as work:
        objs = [os.path.join(work, s + ".o") for s in SOURCES]
        cmds = [[hipcc(), *HIPCC_FLAGS, "-I", os.path.join(HERE, "..", "include"), "-c", os.path.join(CSRC, s), "-o", o]
                for s, o in zip(SOURCES, objs)]
        with ThreadPoolExecutor(max_workers=6) as pool:
            list(pool.map(run, cmds))
        run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", *objs, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
