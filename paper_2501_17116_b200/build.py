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
CALL_PATH = os.path.join(HERE, "_mx_call.so")
SOURCES = ("api.cu", "gemm_fp4.cu", "quantize.cu", "compensate.cu", "wgrad_dense_tc.cu", "mx_api.cu", "mx_quantize.cu",
           "mx_gemm.cu")


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libfp4linear.so")


def needs_build() -> bool:
    if not (os.path.exists(LIB_PATH) and os.path.exists(CALL_PATH)):
        return True
    built = min(os.path.getmtime(LIB_PATH), os.path.getmtime(CALL_PATH))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "fp4_linear.h")]
    return any(os.path.getmtime(d) > built for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """nvcc -> paper_2501_17116_b200/libfp4linear.so.  Returns the library path."""
    if not force and not needs_build():
        return LIB_PATH
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
    _build_call()
    return LIB_PATH


def _build_call():
    """g++ -> paper_2501_17116_b200/_mx_call.so, for the interpreter and the torch that run this."""
    import torch
    from torch.utils import cpp_extension
    dirs = [sysconfig.get_paths()["include"], os.path.join(ROOT, "include")] + cpp_extension.include_paths()
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [a for d in dirs for a in ("-isystem", d)] + [os.path.join(CSRC, "mx_call.cpp"), "-o", CALL_PATH]
    cmd += [a for d in cpp_extension.library_paths() for a in ("-L", d)] + ["-ltorch_python", "-ltorch_cpu", "-lc10"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("g++ failed:\n" + proc.stdout + proc.stderr)


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
