"""Build the C-ABI library (libbcast_b200.so) in-tree with nvcc for sm_100a, and the extension module
that hands torch tensors to its serving operators (_serve_native.so) with the host compiler.

Run as ``python -m paper_1603_06809_b200.build`` or call :func:`build`.  The shared objects are
placed next to this file so that they travel with the source tree.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
REPO_DIR = os.path.dirname(PKG_DIR)
LIB_PATH = os.path.join(PKG_DIR, "libbcast_b200.so")
SOURCES = [os.path.join(PKG_DIR, "csrc", f) for f in ("plan.cpp", "walk_tables.cpp", "shard.cpp", "exec.cu",
                                                    "serve_linear.cu", "serve_attn.cu", "serve_verify.cu")]
HEADERS = [os.path.join(REPO_DIR, "include", f) for f in ("bcast.h", "bcast_serve.h")] + \
          [os.path.join(PKG_DIR, "csrc", f) for f in ("plan_internal.h", "walk_tables.h", "exec_internal.h", "kernels.cuh",
                                                      "serve_internal.h", "serve_tma.h", "serve_device.cuh")]

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-Xcompiler", "-fPIC", "-shared", "-Xlinker", "-soname=libbcast_b200.so", "-I", os.path.join(REPO_DIR, "include"),
]


BIND_PATH = os.path.join(PKG_DIR, "_serve_native.so")
BIND_SOURCES = [os.path.join(PKG_DIR, "csrc", "serve_bind.cpp")]
BIND_HEADERS = [os.path.join(REPO_DIR, "include", f) for f in ("bcast.h", "bcast_serve.h")]


def _older(path: str, sources) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(f) > os.path.getmtime(path) for f in sources)


def needs_build() -> bool:
    return _older(LIB_PATH, SOURCES + HEADERS) or _older(BIND_PATH, BIND_SOURCES + BIND_HEADERS)


def _run(cmd, path: str) -> None:
    """Run a compiler command that ends in the name of its output, and put that in place of ``path``."""
    tmp = path + f".{os.getpid()}.tmp"
    subprocess.check_call([*cmd, "-o", tmp])
    os.replace(tmp, path)


def _build_bind(nvcc: str) -> None:
    import torch
    troot = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(nvcc) or nvcc)))
    include = [os.path.join(REPO_DIR, "include"), os.path.join(troot, "include"), os.path.join(troot, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-DTORCH_API_INCLUDE_EXTENSION_H",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[a for d in include for a in ("-isystem", d)], *BIND_SOURCES,
          LIB_PATH, f"-L{troot}/lib", "-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_python",
          "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{troot}/lib"], BIND_PATH)


def _build_library(nvcc: str, verbose: bool = False) -> None:
    _run([nvcc, *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), *SOURCES], LIB_PATH)


def _nvcc() -> str:
    return os.environ.get("NVCC", "nvcc")


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library and the extension module if they are missing or older than their sources; return the
    library's path."""
    if force or _older(LIB_PATH, SOURCES + HEADERS):
        _build_library(_nvcc(), verbose)
    if force or _older(BIND_PATH, BIND_SOURCES + BIND_HEADERS):
        _build_bind(_nvcc())
    return LIB_PATH


def ensure_built() -> str:
    """Build what is missing or older than its sources; keep what there is when no compiler is at hand.  The library has
    to be there in the end.  The extension module need not: only ``serve`` loads it, and says so if it cannot.
    Returns the path of the library."""
    failed = (OSError, subprocess.CalledProcessError)
    if not os.path.exists(LIB_PATH):
        _build_library(_nvcc())
    elif _older(LIB_PATH, SOURCES + HEADERS):
        try:
            _build_library(_nvcc())
        except failed:
            pass
    if _older(BIND_PATH, BIND_SOURCES + BIND_HEADERS):
        try:
            _build_bind(_nvcc())
        except (*failed, ImportError):                # no compiler, no headers, no torch
            pass
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
