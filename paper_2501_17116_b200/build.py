"""Compile the CUDA sources of this package into one shared library, in-tree, for sm_100a, and the module that calls a part
of it from Python."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libfp4linear.so")
SOURCES = ("api.cu", "gemm_fp4.cu", "quantize.cu", "compensate.cu", "wgrad_dense_tc.cu", "mx_api.cu", "mx_quantize.cu",
           "mx_gemm.cu")


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libfp4linear.so")


def call_path() -> str:
    """Where the module is that hands tensors to the library.  It is built against torch's C++ interface, which changes from version to version, and
    the interpreter's: their names are part of its own, so that one built for others is never loaded."""
    import torch
    built_for = f"torch{torch.__version__}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}-{sysconfig.get_config_var('SOABI')}"
    return os.path.join(HERE, f"_mx_call-{built_for}.so")


def _older(path: str, *sources: str) -> bool:
    if not os.path.exists(path):
        return True
    built = os.path.getmtime(path)
    return any(os.path.getmtime(s) > built for s in sources + (os.path.join(ROOT, "include", "fp4_linear.h"),))


def needs_build() -> bool:
    return _library_is_old() or _call_is_old()


def _library_is_old() -> bool:
    return _older(LIB_PATH, *(os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")))


def _call_is_old() -> bool:
    return _older(call_path(), os.path.join(CSRC, "mx_call.cpp"))


def build(force: bool = False, verbose: bool = False) -> str:
    """nvcc -> paper_2501_17116_b200/libfp4linear.so, g++ -> the module at call_path().  Returns the library path."""
    if force or _library_is_old():
        _build_library(verbose)
    if force or _call_is_old():
        _build_call()
    return LIB_PATH


def _build_library(verbose: bool):
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-shared", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES] + ["-o", LIB_PATH, "-cudart", "static"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + proc.stdout + proc.stderr)
    if verbose:
        print(proc.stdout + proc.stderr)


def _build_call():
    import torch
    from torch.utils import cpp_extension
    dirs = [sysconfig.get_paths()["include"], os.path.join(ROOT, "include")] + cpp_extension.include_paths()
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [a for d in dirs for a in ("-isystem", d)] + [os.path.join(CSRC, "mx_call.cpp"), "-o", call_path()]
    cmd += [a for d in cpp_extension.library_paths() for a in ("-L", d)] + ["-ltorch_python", "-ltorch_cpu", "-lc10"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("g++ failed:\n" + proc.stdout + proc.stderr)


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
