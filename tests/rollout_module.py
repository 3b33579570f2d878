"""rollout.py over the stand-ins of rollout_module_main.cpp.  For a process of its own: torch's idea of the current GPU is replaced in it."""
import ctypes
import importlib.machinery
import importlib.util
import os
import subprocess
import sysconfig

import torch
from torch.utils.cpp_extension import include_paths, library_paths

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def build(folder):
    so = os.path.join(folder, "_rollout.so")
    cmd = ["g++", "-O0", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-DHF_BUILD", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2409_19256_amd", "csrc")]
    for path in include_paths() + [sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", path]
    cmd += [os.path.join(HERE, "rollout_module_main.cpp"), "-o", so]
    for path in library_paths():
        cmd += ["-L", path]
    subprocess.run(cmd + ["-ltorch_python", "-ltorch_cpu", "-lc10"], check=True)
    return so


class Stand:
    """rollout with its native module replaced; tensors, calls and the current device of the stand-ins."""

    def __init__(self, so):
        from paper_2409_19256_amd import binding, rollout
        loader = importlib.machinery.ExtensionFileLoader("_rollout", so)
        native = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_rollout", so, loader=loader))
        loader.exec_module(native)
        native.set_error(binding.HfError)
        rollout._native = native
        rollout._stream_of = lambda device: 1000 + device
        self.rollout, self._lib = rollout, ctypes.PyDLL(so)
        self._lib.stand_in_tensor.restype = self._lib.calls.restype = ctypes.py_object
        self._lib.stand_in_tensor.argtypes = [ctypes.py_object, ctypes.c_int, ctypes.c_int]

    TYPES = {torch.int32: 3, torch.int64: 4, torch.float16: 5, torch.float32: 6, torch.bfloat16: 15}

    def tensor(self, *shape, dtype=torch.bfloat16, device=0):
        return self._lib.stand_in_tensor(shape, self.TYPES[dtype], device)

    def calls(self):
        return self._lib.calls()

    def current_device(self):
        return self._lib.current_device()
