"""Builds libddmerge.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and _ddtorch.so, the
binding of the tensor-list and matrix calls, with g++ against torch's headers."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libddmerge.so")
BINDING = os.path.join(PKG, "_ddtorch.so")
SOURCES = ["dd_merge.cu", "dd_host_stream.cu", "dd_noalloc.cu", "dd_broadcast.cu", "dd_int4.cu", "dd_grad.cu",
           "dd_ffn.cu", "dd_host.cpp"]
NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "--shared", "-Xcompiler", "-fPIC", "-Xptxas", "-v", "-cudart", "static", "--threads", "0",
]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths += [os.path.join(ROOT, "include", f) for f in os.listdir(os.path.join(ROOT, "include"))]
    return max(os.path.getmtime(p) for p in paths)


def _fresh(path: str) -> bool:
    return os.path.exists(path) and os.path.getmtime(path) >= _newest_source_mtime()


def _run(cmd, what: str, verbose: bool) -> None:
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
    if proc.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed building {what}")


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library and the binding if they are missing or older than the sources; returns the
    library's path."""
    if force or not _fresh(LIB):
        _build_library(verbose)
    if force or not _fresh(BINDING):
        _build_binding(verbose)
    return LIB


def _build_library(verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", tmp]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    _run(cmd, "libddmerge.so", verbose)
    os.replace(tmp, LIB)


def _build_binding(verbose: bool) -> None:
    import sysconfig

    import torch
    base = os.path.join(os.path.dirname(torch.__file__))
    tmp = BINDING + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-w",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
           "-I", os.path.join(base, "include"), "-I", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-o", tmp, os.path.join(CSRC, "dd_torch.cpp"), "-L", PKG, "-lddmerge", "-Wl,-rpath,$ORIGIN",
           "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    _run(cmd, "_ddtorch.so", verbose)
    os.replace(tmp, BINDING)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
