"""Builds libhfreshard.so (gfx950) in-tree with hipcc.  Usage: python -m paper_2409_19256_amd.build"""
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
LIB = os.path.join(PKG, "libhfreshard.so")
BENCH_EXE = os.path.join(PKG, "hfbench")
TORCH_MODULE = os.path.join(PKG, "_rollout.so")
SOURCES = ["planner.cpp", "reshard_kernels.hip", "abi.hip", "append_kernels.hip", "attend_kernels.hip", "logprob_kernels.hip", "rollout_abi.hip",
           "adjust_kernels.hip", "distill_kernels.hip", "page_kernels.hip", "steps_abi.hip"]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return exe


def build_library(verbose: bool = True) -> str:
    """Compile every source for gfx950 and link the shared library; returns its path.  rollout.py's native modules are built beside it where they can be."""
    flags = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fvisibility=hidden",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             # kernel arguments arrive in registers: a workgroup here lives for two or three round trips to
             # memory, and without this the first is for the arguments (small calls 2-6 % faster, long ones level)
             "-mllvm", "-amdgpu-kernarg-preload-count=16",
             "-Wall", "-Wno-unused-command-line-argument",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-DHF_BUILD"]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True, cwd=ROOT)

    # a process for each source: one after another they take four minutes
    with tempfile.TemporaryDirectory() as folder, ThreadPoolExecutor(int(os.environ.get("MAX_JOBS", 0)) or os.cpu_count() or 1) as jobs:
        objects = [os.path.join(folder, s + ".o") for s in SOURCES]
        for job in [jobs.submit(run, [hipcc()] + flags + ["-x", "hip", "-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, objects)]:
            job.result()
        run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-Wl,-soname,libhfreshard.so"] + objects + ["-o", LIB + ".tmp"])
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
        build_torch_modules(verbose)
    except (OSError, subprocess.CalledProcessError) as e:
        # no headers of Python's, no host compiler that torch's headers pass: the library does not need them.  An older module would not fit it.
        for module in torch_modules().values():
            if os.path.exists(module):
                os.remove(module)
        print(f"_rollout and _steps were not built, so that paper_2409_19256_amd.rollout cannot be imported: {e}", file=sys.stderr, flush=True)
    return LIB


def torch_modules() -> dict:
    """Source and module of each of rollout.py's native parts; they lie side by side."""
    return {"rollout_torch.cpp": TORCH_MODULE, "steps_torch.cpp": os.path.join(os.path.dirname(TORCH_MODULE), "_steps.so")}


def build_torch_modules(verbose: bool = True) -> None:
    """rollout.py's native part: host code over torch's headers, linked against the library.  Without torch there is nothing to build it for."""
    try:
        import torch
        from torch.utils.cpp_extension import include_paths, library_paths
    except ImportError:
        return
    head = [shutil.which("g++") or hipcc(), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I", os.path.join(ROOT, "include")]
    for path in include_paths() + [sysconfig.get_paths()["include"]]:
        head += ["-isystem", path]
    tail = ["-L", PKG, "-lhfreshard", "-Wl,-rpath,$ORIGIN"]
    for path in library_paths():
        tail += ["-L", path]
    tail += ["-ltorch_python", "-ltorch_cpu", "-lc10"]
    for source, module in torch_modules().items():
        cmd = head + [os.path.join(CSRC, source), "-o", module + ".tmp"] + tail
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True, cwd=ROOT)
        os.replace(module + ".tmp", module)


if __name__ == "__main__":
    build_library()
    print("built", LIB)
    sys.exit(0)
