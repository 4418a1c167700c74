"""Build librkrotor.so (the solver), librkblock.so (operators of the blocks that a schedule
runs) with its Python module _rkblock.so, and librkcalib.so (measured GPU ceilings for the
benchmark), HIP for gfx950, in-tree with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librkrotor.so")
SOURCES = ["rk_api.hip", "rk_kernels.hip", "rk_tile.hip", "rk_host.cpp"]
CALIB_LIB = os.path.join(PKG, "librkcalib.so")
CALIB_SOURCES = ["rk_calib.hip"]
BLOCK_LIB = os.path.join(PKG, "librkblock.so")
BLOCK_SOURCES = ["rkb_norm.hip", "rkb_ckpt.hip", "rkb_gemm.hip", "rkb_attn.hip", "rkb_attn_bwd.hip", "rkb_attn_api.hip",
                 "rkb_kv8.hip"]
# Sums of the attention kernels stay in vector registers past 256 of them, where vector instructions reach them: kept in the
# accumulation registers, they are copied to and fro.  Heads of 256 columns gain most (one query over 16 x 4096 tokens of 4 key
# heads takes 60 us instead of 195), the others are the same or a few percent faster.
SOURCE_FLAGS = {s: ["-mllvm", "-amdgpu-mfma-vgpr-form=1"] for s in ("rkb_attn.hip", "rkb_attn_bwd.hip")}
BIND_LIB = os.path.join(PKG, "_rkblock.so")
BIND_SOURCE = "rkb_bind.cpp"
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


def _run(cmd, out: str, verbose: bool) -> str:
    if verbose:
        print(" ".join([*cmd, "-o", out]), flush=True)
    res = subprocess.run([*cmd, "-o", out + ".tmp"], capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed ({res.returncode})")
    os.replace(out + ".tmp", out)
    return out


def _compile(sources, out: str, verbose: bool) -> str:
    """Every source to an object of its own, side by side (a single call of hipcc takes them in turn), then linked."""
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(os.cpu_count()) as pool:
        flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        objects = list(pool.map(lambda s: _run([hipcc(), *flags, *SOURCE_FLAGS.get(s, []), "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
                                                os.path.join(CSRC, s)], os.path.join(tmp, s + ".o"), verbose), sources))
        return _run([hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objects], out, verbose)


def _compile_binding(verbose: bool) -> str:
    """The Python module that marshals tensors for librkblock: host code, against torch's headers and
    libraries (and so torch's HIP runtime)."""
    import torch
    tdir = os.path.dirname(torch.__file__)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(hipcc())))
    if not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime_api.h")):
        rocm = "/opt/rocm"
    return _run([os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__",
                 "-DUSE_ROCM", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                 "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(tdir, "include"),
                 "-isystem", os.path.join(rocm, "include"), "-isystem", sysconfig.get_paths()["include"],
                 os.path.join(CSRC, BIND_SOURCE), "-L", PKG, "-lrkblock", "-L", os.path.join(tdir, "lib"),
                 "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip", "-lamdhip64",
                 "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{os.path.join(tdir, 'lib')}"], BIND_LIB, verbose)


def build(verbose: bool = False) -> str:
    """All libraries; returns the solver's path."""
    _compile(BLOCK_SOURCES, BLOCK_LIB, verbose)
    _compile_binding(verbose)
    _compile(CALIB_SOURCES, CALIB_LIB, verbose)
    return _compile(SOURCES, LIB, verbose)


if __name__ == "__main__":
    print(build(verbose=True))
