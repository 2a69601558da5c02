"""Builds in-tree the C-ABI CUDA library ``libnereus.so`` with nvcc, for sm_100a only, and the torch-facing marshalling
``_nereus_torch.so`` of ``logits.py`` with g++ (host code, linked against the library)."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libnereus.so")
EXT_SRC = os.path.join(HERE, "torch_ext", "nereus_torch.cpp")
EXT = os.path.join(HERE, "_nereus_torch.so")


def sources() -> list:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    deps = sources() + glob.glob(os.path.join(CSRC, "*.hpp")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > os.path.getmtime(LIB) for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        build_ext(force)
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC,-Wall,-Wextra", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", tmp] + (["-Xptxas", "-v"] if verbose else []) + sources()
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    build_ext(force)
    return LIB


def build_ext(force: bool = False) -> str:
    header = os.path.join(ROOT, "include", "nereus.h")
    if not force and os.path.exists(EXT) and all(os.path.getmtime(d) <= os.path.getmtime(EXT) for d in (EXT_SRC, header)):
        return EXT
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), sysconfig.get_paths()["include"], os.path.join(base, "include"),
               os.path.join(base, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    tmp = EXT + f".tmp{os.getpid()}"
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-o", tmp, EXT_SRC]
                          + [x for i in include for x in ("-isystem", i)]
                          + ["-L", HERE, "-lnereus", "-Wl,-rpath,$ORIGIN", "-L", os.path.join(base, "lib"), "-ltorch_python",
                             "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    os.replace(tmp, EXT)
    return EXT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
