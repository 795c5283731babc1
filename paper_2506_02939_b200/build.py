"""Compile the CUDA library in-tree for sm_100a with nvcc, and the binding of its training operators with g++ (no GPU needed)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libpamm_b200.so"

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC",
]


def _sources():
    return sorted(CSRC.glob("*.cu")) + sorted(CSRC.glob("*.cuh")) + [PKG.parent / "include" / "pamm.h"]


def binding_path() -> Path:
    """The binding for this Python and this torch: its name has both, so that one built for others is not taken for it."""
    import torch
    return PKG / f"_binding-torch{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}"


def _build_binding(force: bool) -> None:
    import torch
    binding, source, header = binding_path(), CSRC / "binding.cpp", PKG.parent / "include" / "pamm.h"
    newest = max(source.stat().st_mtime, header.stat().st_mtime)
    if not force and binding.exists() and binding.stat().st_mtime >= newest:
        return
    root = Path(torch.__file__).resolve().parent
    cuda = Path(os.environ.get("CUDA_HOME", "/usr/local/cuda"))
    tmp = PKG / f"_binding.{os.getpid()}.tmp"
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f"-I{root / 'include'}", f"-I{root / 'include' / 'torch' / 'csrc' / 'api' / 'include'}",
           f"-I{sysconfig.get_paths()['include']}", f"-I{cuda / 'include'}", "-o", str(tmp), str(source),
           f"-L{PKG}", "-l:libpamm_b200.so", f"-L{root / 'lib'}", "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10",
           "-Wl,-rpath,$ORIGIN"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, binding)


def build(force: bool = False, verbose: bool = False) -> Path:
    _build_library(force, verbose)
    _build_binding(force)
    return LIB


def _build_library(force: bool, verbose: bool) -> None:
    newest = max(p.stat().st_mtime for p in _sources())
    if not force and LIB.exists() and LIB.stat().st_mtime >= newest:
        return
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = LIB.with_suffix(f".{os.getpid()}.tmp")
    cmd = [nvcc, *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-o", str(tmp), str(CSRC / "pamm_lib.cu")]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
