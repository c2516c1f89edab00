"""Builds the CUDA library (libcrisp.so) in-tree with nvcc for sm_100a, and the compiled part of the binding (_calls.*.so)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcrisp.so")
SOURCES = ["api.cu", "route.cu", "select.cu", "prefill.cu", "cache_pages.cu", "cache_attention.cu", "cache_prefill.cu",
           "cache_join.cu", "norm.cu", "matmul.cu", "matmul_pair.cu", "rotary.cu", "selftest.cu"]
HEADERS = ["common.cuh", "cache.cuh", "cache_split.cuh", "cache_codes.cuh", "cache_ring.h", "operand.cuh", "matmul.cuh", "matmul_wait.h",
           "softmax_rows.cuh", "sm100_ptx.cuh", os.path.join("..", "..", "include", "crisp.h")]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def calls_path() -> str:
    """The compiled part of the binding uses torch's and Python's C++ and C interfaces, which differ between versions: its name
    says for which ones it was built, so that others do not load it."""
    import torch
    return os.path.join(HERE, f"_calls.{sys.implementation.cache_tag}-torch-{torch.__version__}.so")


def needs_build() -> bool:
    calls = calls_path()
    if not os.path.exists(LIB) or not os.path.exists(calls):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(calls))
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS + ["calls.cpp"]] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu for sm_100a into one shared library; returns its path."""
    if not force and not needs_build():
        return LIB
    cmd = [_nvcc(), "-shared", "-Xcompiler", "-fPIC", "-O3", "-std=c++17", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static",
           "-o", LIB] + [os.path.join(CSRC, f) for f in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libcrisp.so")
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    build_calls()
    return LIB


def build_calls() -> str:
    """Compile calls.cpp against the torch that is installed; returns the module's path."""
    import torch
    path = calls_path()
    torch_dir = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda"
    include = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-o", path, os.path.join(CSRC, "calls.cpp")] + [f"-I{d}" for d in include] + [f"-L{os.path.join(torch_dir, 'lib')}"] + [
           f"-l{x}" for x in ("torch", "torch_cpu", "torch_cuda", "torch_python", "c10", "c10_cuda")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed building the compiled part of the binding")
    return path


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
