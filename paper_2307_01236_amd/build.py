"""Build librkrotor.so (the solver), librkblock.so (operators of the blocks that a schedule
runs) and librkcalib.so (measured GPU ceilings for the benchmark), HIP for gfx950, in-tree
with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librkrotor.so")
SOURCES = ["rk_api.hip", "rk_kernels.hip", "rk_tile.hip", "rk_host.cpp"]
CALIB_LIB = os.path.join(PKG, "librkcalib.so")
CALIB_SOURCES = ["rk_calib.hip"]
BLOCK_LIB = os.path.join(PKG, "librkblock.so")
BLOCK_SOURCES = ["rkb_norm.hip", "rkb_ckpt.hip", "rkb_gemm.hip"]
ARCH = "gfx950"

HIPCC_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Wno-unused-command-line-argument",
    # keep the compiler from emitting packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # preload a kernel's leading scalar arguments into SGPRs at wave start (as many as fit;
    # none for kernels whose first argument is a struct); the finalize is laid out for it
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _compile(sources, out: str, verbose: bool) -> str:
    srcs = [os.path.join(CSRC, s) for s in sources]
    tmp = out + ".tmp"
    cmd = [hipcc(), *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, *srcs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"hipcc failed ({res.returncode})")
    os.replace(tmp, out)
    return out


def build(verbose: bool = False) -> str:
    """All three libraries; returns the solver's path."""
    _compile(BLOCK_SOURCES, BLOCK_LIB, verbose)
    _compile(CALIB_SOURCES, CALIB_LIB, verbose)
    return _compile(SOURCES, LIB, verbose)


if __name__ == "__main__":
    print(build(verbose=True))
