"""Build the HIP libraries for gfx950 with hipcc: libdecomoe.so (the sources
of csrc/, the MoE layers) and libdecomoe_block.so (the sources of csrc/block/,
the attention half of a block).

Run as ``python -m paper_2609_38823_amd.build``; the libraries are written
in-tree next to this file so that they travel with the source tree.
"""

from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libdecomoe.so")
BLOCK_LIB = os.path.join(HERE, "libdecomoe_block.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    # no packed-fp32 instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep per-thread arrays in registers instead of silently moving them to LDS
    "-mllvm", "-disable-promote-alloca-to-lds",
    "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))


def block_sources() -> list[str]:
    return sorted(glob.glob(os.path.join(HERE, "csrc", "block", "*.hip")))


def build(verbose: bool = False) -> str:
    """Compile every HIP source into the two shared libraries (at the same
    time); returns the path of libdecomoe.so."""
    jobs = []
    for lib, files in ((LIB, sources()), (BLOCK_LIB, block_sources())):
        cmd = [hipcc(), *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), *files, "-o", lib + ".tmp"]
        jobs.append((lib, cmd, subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True)))
    noise = "is not a recognized feature for this target"
    failed = []
    for lib, cmd, job in jobs:
        err = job.communicate()[1]
        errs = "\n".join(l for l in (err or "").splitlines() if noise not in l)
        if job.returncode != 0:
            failed.append(f"hipcc failed ({job.returncode}):\n{' '.join(cmd)}\n{errs}")
            continue
        if verbose and errs.strip():
            print(errs, file=sys.stderr)
        os.replace(lib + ".tmp", lib)
    if failed:
        raise RuntimeError("\n".join(failed))
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
