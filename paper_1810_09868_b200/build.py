"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache)."""
from __future__ import annotations

import glob
import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libvgg19_b200.so")
CALLS_SOURCE = os.path.join(CSRC, "tensor_calls.cpp")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "--threads", "0"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu"))) + [os.path.join(ROOT, "seeded_inputs", "seeded_inputs.c")]


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libvgg19_b200.so next to this file."""
    if force or _stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + sources()
        subprocess.run(cmd, check=True)
    build_calls(force)
    return LIB


def calls_path() -> str:
    """The compiled calls of this interpreter and this torch: they read torch's own objects, whose layout is no interface."""
    import sys

    import torch
    tag = f"{sys.implementation.cache_tag}-torch{torch.__version__}-{(torch.version.git_version or 'local')[:8]}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}"
    return os.path.join(PKG, f"_tensor_calls.{tag}.so")


def build_calls(force: bool = False) -> str:
    """Compile csrc/tensor_calls.cpp, which reads torch tensors, against the installed torch's headers."""
    deps = (CALLS_SOURCE, os.path.join(ROOT, "include", "vgg19_b200.h"))
    path = calls_path()
    if force or not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps):
        import sysconfig

        import torch
        where = os.path.dirname(torch.__file__)
        cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
        include = (os.path.join(where, "include"), os.path.join(where, "include", "torch", "csrc", "api", "include"),
                   os.path.join(cuda, "include"), sysconfig.get_paths()["include"])
        cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
        for i in include:
            cmd += ["-isystem", i]
        made = f"{path}.{os.getpid()}"
        cmd += ["-o", made, CALLS_SOURCE, "-L" + os.path.join(where, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda",
                "-L" + PKG, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]
        subprocess.run(cmd, check=True)
        os.replace(made, path)  # (a process that has the old one open keeps it)
    return path
