"""Compile the CUDA sources into libdnns.so (in-tree) with nvcc for sm_100a, and the calls from torch tensors into _native.so."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libdnns.so")
LIB_CHECKED = os.path.join(HERE, "libdnns_checked.so")   # -DDNNS_BOUNDS_CHECK: data-dependent indices verified
NATIVE = os.path.join(HERE, "_native.so")                 # calls on rows in 8 bits straight from torch tensors
NATIVE_KEY = os.path.join(HERE, "_native.key")            # the torch and Python that it was built for
NATIVE_SOURCE = os.path.join(HERE, "csrc", "torch_binding.cpp")
SOURCES = sorted(glob.glob(os.path.join(HERE, "csrc", "*.cu")))
HEADERS = sorted(glob.glob(os.path.join(HERE, "csrc", "*.cuh"))) + [os.path.join(ROOT, "include", "dnns.h")]


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(f) > t for f in SOURCES + HEADERS)


def native_key() -> str:
    """What a built _native.so depends on beside its sources."""
    import torch
    return f"torch {torch.__version__} cxx11abi {int(torch._C._GLIBCXX_USE_CXX11_ABI)} {sysconfig.get_config_var('SOABI')}\n"


def native_needs_build() -> bool:
    if not os.path.exists(NATIVE) or not os.path.exists(NATIVE_KEY):
        return True
    t = os.path.getmtime(NATIVE)
    if any(os.path.getmtime(f) > t for f in (NATIVE_SOURCE, os.path.join(ROOT, "include", "dnns.h"))):
        return True
    with open(NATIVE_KEY) as f:
        return f.read() != native_key()


def build_native(force: bool = False) -> str:
    if not force and not native_needs_build():
        return NATIVE
    import torch
    top = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
                           "-isystem", os.path.join(top, "include"), "-isystem", os.path.join(top, "include", "torch", "csrc", "api", "include"),
                           "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"],
                           "-o", NATIVE, NATIVE_SOURCE, "-L", os.path.join(top, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"])
    with open(NATIVE_KEY, "w") as f:
        f.write(native_key())
    return NATIVE


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """libdnns.so and _native.so.  checked: the test-only variant whose kernels verify every data-dependent index (libdnns_checked.so)."""
    lib = LIB_CHECKED if checked else LIB
    build_native(force)
    if not force and not needs_build(lib):
        return lib
    nvcc = os.environ.get("NVCC", "nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared",
           "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-o", lib] + SOURCES
    if checked:
        cmd.insert(1, "-DDNNS_BOUNDS_CHECK")
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
