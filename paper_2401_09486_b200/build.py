"""Builds libloma.so (the C-ABI CUDA library, nvcc for sm_100a) and _marshal.so (argument marshalling for its shortest calls from
Python, g++ against torch's headers) in-tree.  The library needs nothing but CUDA."""

from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig
import warnings

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(PKG_DIR, "libloma.so")
MARSHAL_SRC = os.path.join(CSRC, "marshal.cpp")
MARSHAL_PATH = os.path.join(PKG_DIR, "_marshal.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-lineinfo", "-O3", "-std=c++17",
    "--shared", "-Xcompiler", "-fPIC",
    "-Xcompiler", "-fvisibility=hidden",
]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return cand


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _older(path: str, deps) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(p) > os.path.getmtime(path) for p in deps)


def _run(cmd, what: str, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{what} failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr, file=sys.stderr)


def marshal_key() -> str:
    """What _marshal.so has to have been built for: it uses torch's C++ classes, whose layout changes between versions."""
    import torch

    return f"python {sys.version_info[0]}.{sys.version_info[1]}, torch {torch.__version__}, C++ ABI {int(torch._C._GLIBCXX_USE_CXX11_ABI)}"


def _marshal_stale() -> bool:
    if _older(MARSHAL_PATH, [MARSHAL_SRC, os.path.join(INCLUDE, "loma.h")]):
        return True
    with open(MARSHAL_PATH, "rb") as f:
        return marshal_key().encode() + b"\0" not in f.read()


def build_marshal(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/marshal.cpp into the extension module if it is out of date, or was built for another torch; returns its path."""
    if not force and not _marshal_stale():
        return MARSHAL_PATH
    import torch

    if os.path.exists(MARSHAL_PATH):
        os.remove(MARSHAL_PATH)      # where the build fails, none is better than one for another torch
    root = os.path.dirname(os.path.abspath(torch.__file__))
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    includes = [INCLUDE, os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    lib = os.path.join(root, "lib")
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DLOMA_BUILT_FOR="{marshal_key()}"', *[f"-I{d}" for d in includes], MARSHAL_SRC, "-o", MARSHAL_PATH,
           f"-L{lib}", f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    _run(cmd, "g++", verbose)
    return MARSHAL_PATH


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every csrc/*.cu into one shared library and, for its users from Python, csrc/marshal.cpp into the extension module;
    returns the library's path.  Without torch or a C++ compiler there is the library alone, for C programs, and a warning."""
    if force or _older(LIB_PATH, sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))):
        cmd = [_nvcc(), *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC, "-o", LIB_PATH, *sources()]
        if verbose:
            cmd[1:1] = ["-Xptxas", "-v"]
        _run(cmd, "nvcc", verbose)
    try:
        build_marshal(force, verbose)
    except (ImportError, OSError, RuntimeError) as e:
        warnings.warn(f"{LIB_PATH} is built, the extension module for Python is not: {e}", stacklevel=2)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
