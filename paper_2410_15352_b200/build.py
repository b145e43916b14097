"""Builds libcompact.so (sm_100a) in-tree with nvcc, and the Python module of the block operators with g++."""
from __future__ import annotations

import os
import subprocess
import sysconfig
import warnings

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.environ.get("COMPACT_LIB", os.path.join(PKG_DIR, "libcompact.so"))
SOURCES = ["compact_api.cu", "block_api.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-shared",
]


# Python side of the block operators: a plain C++ module over torch's headers, no device code
MODULE_PATH = os.path.join(PKG_DIR, "_block_py.so")
MODULE_SOURCE = os.path.join(CSRC, "block_py.cpp")
MODULE_HEADERS = [os.path.join(os.path.dirname(PKG_DIR), "include", h) for h in ("compact.h", "compact_block.h")]


def _newest_source_mtime() -> float:
    newest = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(PKG_DIR), "include")):
        for f in os.listdir(root):
            newest = max(newest, os.path.getmtime(os.path.join(root, f)))
    return newest


def module_tag() -> str:
    """What a module works with: this Python and this torch.  It carries the tag it was built with."""
    import torch

    return f"python {sysconfig.get_config_var('SOABI')}, torch {torch.__version__}, abi {int(torch._C._GLIBCXX_USE_CXX11_ABI)}"


def module_fits() -> bool:
    """Whether there is a module, built for this Python and this torch."""
    if not os.path.exists(MODULE_PATH):
        return False
    with open(MODULE_PATH, "rb") as f:
        return f"built for [{module_tag()}]".encode() in f.read()


def _module_command(out: str) -> list:
    import torch

    home, cuda = os.path.dirname(torch.__file__), os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f'-DBUILT_FOR="{module_tag()}"',
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + sysconfig.get_paths()["include"]]
    cmd += ["-isystem" + p for p in (home + "/include", home + "/include/torch/csrc/api/include", cuda + "/include")]
    cmd += [MODULE_SOURCE, "-L" + home + "/lib", "-L" + cuda + "/lib64"]
    return cmd + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python", "-ldl", "-o", out]


def build_module(force: bool = False) -> str:
    """Compiles the Python module unless it is up to date and fits this Python and torch."""
    newest = max(os.path.getmtime(f) for f in (MODULE_SOURCE, *MODULE_HEADERS))
    if not force and module_fits() and os.path.getmtime(MODULE_PATH) >= newest:
        return MODULE_PATH
    # beside it and then in its place: a process that has the old one loaded keeps it
    part = f"{MODULE_PATH}.{os.getpid()}"
    try:
        proc = subprocess.run(_module_command(part), capture_output=True, text=True)
        if proc.returncode != 0:
            raise RuntimeError("g++ failed:\n" + proc.stdout + proc.stderr)
        os.replace(part, MODULE_PATH)
    finally:
        if os.path.exists(part):
            os.remove(part)
    return MODULE_PATH


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles the CUDA sources into libcompact.so, and the Python module beside it, unless they are up to date.

    The C ABI needs nvcc alone.  Where the module cannot be built (no torch headers, no C++ compiler) the library stands all the same: the
    reason is given as a warning, and `block` raises when it is used."""
    path = _build_cuda(force, verbose)
    try:
        build_module(force)
    except (ImportError, OSError, RuntimeError) as e:
        warnings.warn(f"libcompact.so is built, the Python module of the block operators is not: {e}", RuntimeWarning, stacklevel=2)
    return path


def _build_cuda(force: bool, verbose: bool) -> str:
    if not force and os.path.exists(LIB_PATH) and os.path.getmtime(LIB_PATH) >= _newest_source_mtime():
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "nvcc")
    cmd = [nvcc, *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
           *[os.path.join(CSRC, s) for s in SOURCES], "-o", LIB_PATH]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + proc.stdout + proc.stderr)
    if verbose:
        print(proc.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
