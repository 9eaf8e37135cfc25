"""Builds libgqla.so (the C-ABI CUDA library, nvcc for sm_100a) and _marshal.so (argument checks for the binding, g++) in-tree."""
from __future__ import annotations

import importlib.metadata
import importlib.util
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


def _nvcc() -> str:
    return os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def _marshal_stamp() -> bytes:
    """What the extension holds of the torch and the Python that it was compiled for (marshal.cpp)."""
    return f"built for torch {importlib.metadata.version('torch').split('+')[0]}, Python {sys.version_info[0]}.{sys.version_info[1]};".encode()


def marshal_fits() -> bool:
    """Whether the extension that is there was compiled for this torch and Python."""
    with open(MARSHAL_PATH, "rb") as f:
        return _marshal_stamp() in f.read()


def _marshal_is_current(sources: list[str]) -> bool:
    return os.path.exists(MARSHAL_PATH) and os.path.getmtime(MARSHAL_PATH) >= max(os.path.getmtime(f) for f in sources) and marshal_fits()


def build_marshal(force: bool = False) -> str:
    """Compiles the Python extension of the binding if it is missing, older than its sources, or was compiled for another torch or
    Python; returns its path."""
    sources = [os.path.join(CSRC, "marshal.cpp"), os.path.join(os.path.dirname(PKG_DIR), "include", "gqla.h")]
    if not force and _marshal_is_current(sources):
        return MARSHAL_PATH
    root = os.path.dirname(importlib.util.find_spec("torch").origin)
    part = f"{MARSHAL_PATH}.{os.getpid()}"  # (a process that has the old one loaded keeps it)
    include = [sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include"), os.path.join(root, "include"),
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
    """Compiles the library if it is missing or older than its sources, and the binding's extension likewise; returns the library's
    path.  The library comes first and needs no Python package; where torch is not installed (nor the binding of use) it is all.
    debug: the -DGQLA_DEBUG build (libgqla_debug.so), whose decode kernels check their piece and tile indices and
    record a violated check in the status word instead of trapping."""
    lib_path = DEBUG_LIB_PATH if debug else LIB_PATH
    if force or not os.path.exists(lib_path) or os.path.getmtime(lib_path) < _newest_source_mtime():
        _build_library(lib_path, verbose, debug)
    if importlib.util.find_spec("torch") is not None:
        build_marshal(force)
    return lib_path


def _build_library(lib_path: str, verbose: bool, debug: bool) -> None:
    cmd = [_nvcc(), *NVCC_FLAGS, *(["-DGQLA_DEBUG"] if debug else []), "-o", lib_path, *[os.path.join(CSRC, s) for s in SOURCES]]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
