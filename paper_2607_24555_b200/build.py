"""Build liblocks.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and then _calls.so, the native marshalling of the calls around
a decode step, with g++ and torch's headers.  The library does without the second: a machine that lacks what it takes builds the first alone."""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblocks.so")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + [os.path.join(ROOT, "include", "locks.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def calls_stale() -> bool:
    """Older than its sources, or built for another torch or Python."""
    from .binding import calls_path, calls_stamp
    path = calls_path()
    if not os.path.exists(path):
        return True
    if any(os.path.getmtime(f) > os.path.getmtime(path) for f in (os.path.join(CSRC, "calls.cpp"), os.path.join(ROOT, "include", "locks.h"))):
        return True
    with open(path, "rb") as f:
        return calls_stamp().encode() not in f.read()


def build_calls(force: bool = False) -> str:
    import sysconfig

    import torch

    from .binding import calls_path, calls_stamp
    out, src = calls_path(), os.path.join(CSRC, "calls.cpp")
    if not force and not calls_stale():
        return out
    t = os.path.dirname(torch.__file__)
    if not shutil.which("g++") or not os.path.exists(os.path.join(t, "include", "c10", "cuda", "CUDAGuard.h")):
        sys.stderr.write("_calls.so is not built: it takes g++ and torch's headers (rotary positions, appends and the 8-bit cache then have no Python calls)\n")
        if os.path.exists(out):   # (a stale one may lay the library's structures out otherwise)
            os.remove(out)
        return ""
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    inc = [os.path.join(ROOT, "include"), os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
           os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DLOCKS_CALLS_STAMP="{calls_stamp()}"'] + [x for i in inc for x in ("-I", i)] + ["-o", out, src, "-L", os.path.join(t, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    return out


def build(force: bool = False, verbose: bool = False) -> str:
    lib = build_library(force, verbose)
    build_calls(force)
    return lib


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
          ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", LIB] + sources()
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose:
        sys.stderr.write(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
