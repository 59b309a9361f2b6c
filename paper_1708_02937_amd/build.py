"""Build libsdnn.so (the HIP kernels and the host runtime of the C ABI) for gfx950, and _tensors.so (the calls on torch
tensors over it, host code), in-tree."""

from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsdnn.so")
TENSORS = os.path.join(HERE, "_tensors.so")
SOURCES = ["setup.hip", "spmm.hip", "resident.hip", "gemm.hip", "spgemm.hip", "semiring.hip", "blocked.hip", "quantize.hip", "route.hip",
           "product8.hip", "tile8.hip", "groups4.hip", "layer.hip", "sample.hip",
           "api.cpp", "operators.cpp"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # packed fp32 instructions stay off: the compiler must not emit them
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    if src.endswith(".cpp"):
        cmd[1:1] = ["-x", "hip"]
    subprocess.run(cmd, check=True)
    return obj


def _compile_tensors() -> str:
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    obj = os.path.join(BUILD, "tensors.o")
    flags = ["-O2", "-std=c++17", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
             "-I", os.path.join(ROOT, "include"), "-isystem", sysconfig.get_paths()["include"]]
    for path in cpp_extension.include_paths():
        flags += ["-isystem", path]
    subprocess.run([CXX, *flags, "-c", os.path.join(CSRC, "tensors.cpp"), "-o", obj], check=True)
    return obj


def _link_tensors(obj: str) -> None:
    from torch.utils import cpp_extension

    tmp = TENSORS + ".tmp"
    libs = [f"-L{p}" for p in cpp_extension.library_paths()] + ["-ltorch_cpu", "-ltorch_python", "-lc10"]
    subprocess.run([CXX, "-shared", "-o", tmp, obj, f"-L{HERE}", "-l:libsdnn.so", *libs, "-Wl,-rpath,$ORIGIN"],
                   check=True)
    os.replace(tmp, TENSORS)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        tensors = ex.submit(_compile_tensors)
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs], check=True)
    os.replace(tmp, LIB)
    _link_tensors(tensors.result())
    if verbose:
        print("built", LIB, TENSORS)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
