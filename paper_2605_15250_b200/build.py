"""Builds libgqla.so (the C-ABI CUDA library, nvcc for sm_100a) and _marshal.so (argument checks for the binding, g++) in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libgqla.so")
SOURCES = ["gqla_api.cu", "gqla_noalloc.cu", "gqla_fp8_paged.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--expt-relaxed-constexpr", "--threads", "0", "-shared", "-Xcompiler", "-fPIC", "-cudart", "static",
]


def _newest_source_mtime() -> float:
    t = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(PKG_DIR), "include")):
        for f in os.listdir(root):
            t = max(t, os.path.getmtime(os.path.join(root, f)))
    return t


MARSHAL_PATH = os.path.join(PKG_DIR, "_marshal.so")


def build_marshal(force: bool = False) -> str:
    """Compiles the Python extension of the binding if it is missing or older than its sources; returns its path."""
    sources = [os.path.join(CSRC, "marshal.cpp"), os.path.join(os.path.dirname(PKG_DIR), "include", "gqla.h")]
    if not force and os.path.exists(MARSHAL_PATH) and os.path.getmtime(MARSHAL_PATH) >= max(os.path.getmtime(f) for f in sources):
        return MARSHAL_PATH
    import torch

    root = os.path.dirname(torch.__file__)
    part = f"{MARSHAL_PATH}.{os.getpid()}"  # (a process that has the old one loaded keeps it)
    include = [sysconfig.get_paths()["include"], "/usr/local/cuda/include", os.path.join(root, "include"),
               os.path.join(root, "include", "torch", "csrc", "api", "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", *(f"-I{d}" for d in include), "-o", part,
           sources[0], "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python",
           "-Wl,--exclude-libs,libstdc++.a"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    os.replace(part, MARSHAL_PATH)
    return MARSHAL_PATH


DEBUG_LIB_PATH = os.path.join(PKG_DIR, "libgqla_debug.so")


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compiles the library if it is missing or older than its sources; returns its path.
    debug: the -DGQLA_DEBUG build (libgqla_debug.so), whose decode kernels check their piece and tile indices and
    record a violated check in the status word instead of trapping."""
    build_marshal(force)
    lib_path = DEBUG_LIB_PATH if debug else LIB_PATH
    if not force and os.path.exists(lib_path) and os.path.getmtime(lib_path) >= _newest_source_mtime():
        return lib_path
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, *NVCC_FLAGS, *(["-DGQLA_DEBUG"] if debug else []), "-o", lib_path, *[os.path.join(CSRC, s) for s in SOURCES]]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)
    return lib_path


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
