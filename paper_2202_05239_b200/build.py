"""Builds the CUDA library (``libf8net.so``) in-tree with nvcc for sm_100a, and the torch binding beside it with g++."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libf8net.so")
BINDING = os.path.join(HERE, "_f8torch.so")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _newest_source_mtime() -> float:
    files = sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh"))
    files.append(os.path.join(os.path.dirname(HERE), "include", "f8net.h"))
    return max(os.path.getmtime(f) for f in files)


def binding_made_for() -> str:
    """The Python and the torch that the binding is bound to: the module holds this text."""
    import torch
    return "made for %s, torch %s;" % (sysconfig.get_config_var("SOABI"), torch.__version__)


def binding_is_current() -> bool:
    """Whether the module is there, newer than what it is made of and made for this Python and this torch."""
    made_of = [os.path.join(CSRC, "f8_torch.cpp"), os.path.join(os.path.dirname(HERE), "include", "f8net.h")]
    if not os.path.exists(BINDING) or os.path.getmtime(BINDING) < max(os.path.getmtime(f) for f in made_of):
        return False
    with open(BINDING, "rb") as f:
        return binding_made_for().encode() in f.read()


def build_binding(force: bool = False) -> str:
    """The calls on torch tensors that are made from C++ (csrc/f8_torch.cpp), linked against torch and the library."""
    if not force and binding_is_current():
        return BINDING
    import torch
    source = os.path.join(CSRC, "f8_torch.cpp")
    at = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    tmp = BINDING + ".tmp%d" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-o", tmp, source,
                           '-DF8_MADE_FOR="%s"' % binding_made_for(),
                           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
                           "-I" + os.path.join(at, "include"), "-I" + os.path.join(at, "include", "torch", "csrc", "api", "include"),
                           "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(cuda, "include"),
                           "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
                           "-L" + HERE, "-l:libf8net.so", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, BINDING)
    return BINDING


def build(force: bool = False, verbose: bool = False) -> str:
    build_library(force, verbose)
    build_binding(force)
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "--threads", "8", "-Xcompiler", "-fPIC", "-shared", "-o", tmp] + sources()
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
