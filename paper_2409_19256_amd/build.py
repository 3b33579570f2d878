"""Builds libhfreshard.so (gfx950) in-tree with hipcc.  Usage: python -m paper_2409_19256_amd.build"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libhfreshard.so")
BENCH_EXE = os.path.join(PKG, "hfbench")
TORCH_MODULE = os.path.join(PKG, "_rollout.so")
SOURCES = ["planner.cpp", "reshard_kernels.hip", "abi.hip", "append_kernels.hip", "attend_kernels.hip", "logprob_kernels.hip", "rollout_abi.hip"]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return exe


def build_library(verbose: bool = True) -> str:
    """Compile every source for gfx950 and link the shared library; returns its path.  rollout.py's native module is built beside it where it can be."""
    cmd = [hipcc(), "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared", "-fvisibility=hidden", "-Wl,-soname,libhfreshard.so",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           # kernel arguments arrive in registers: a workgroup here lives for two or three round trips to
           # memory, and without this the first is for the arguments (small calls 2-6 % faster, long ones level)
           "-mllvm", "-amdgpu-kernarg-preload-count=16",
           "-Wall", "-Wno-unused-command-line-argument",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-DHF_BUILD",
           "-x", "hip"] + [os.path.join(CSRC, s) for s in SOURCES] + ["-o", LIB + ".tmp"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True, cwd=ROOT)
    os.replace(LIB + ".tmp", LIB)
    # hfbench: native driver of the C ABI for rocprofv3 runs (no Python in the traced process)
    cmd = [hipcc(), "-O2", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-Wall", "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"),
           "-x", "hip", os.path.join(CSRC, "hfbench.cpp"), "-x", "none", "-L", PKG, "-lhfreshard", "-Wl,-rpath,$ORIGIN", "-o", BENCH_EXE + ".tmp"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True, cwd=ROOT)
    os.replace(BENCH_EXE + ".tmp", BENCH_EXE)
    try:
        build_torch_module(verbose)
    except (OSError, subprocess.CalledProcessError) as e:
        # no headers of Python's, no host compiler that torch's headers pass: the library does not need them.  An older module would not fit it.
        if os.path.exists(TORCH_MODULE):
            os.remove(TORCH_MODULE)
        print(f"_rollout was not built, so that paper_2409_19256_amd.rollout cannot be imported: {e}", file=sys.stderr, flush=True)
    return LIB


def build_torch_module(verbose: bool = True) -> None:
    """rollout.py's native part: host code over torch's headers, linked against the library.  Without torch there is nothing to build it for."""
    try:
        import torch
        from torch.utils.cpp_extension import include_paths, library_paths
    except ImportError:
        return
    cmd = [shutil.which("g++") or hipcc(), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I", os.path.join(ROOT, "include")]
    for path in include_paths() + [sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", path]
    cmd += [os.path.join(CSRC, "rollout_torch.cpp"), "-o", TORCH_MODULE + ".tmp", "-L", PKG, "-lhfreshard", "-Wl,-rpath,$ORIGIN"]
    for path in library_paths():
        cmd += ["-L", path]
    cmd += ["-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True, cwd=ROOT)
    os.replace(TORCH_MODULE + ".tmp", TORCH_MODULE)


if __name__ == "__main__":
    build_library()
    print("built", LIB)
    sys.exit(0)
