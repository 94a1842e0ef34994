"""Build the CUDA library ``libzgr.so`` in-tree with nvcc for sm_100a, and beside it ``_zgr_bind-<torch>-<python>.so``, the marshalling of
the forward-pass operators from torch tensors."""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libzgr.so")
SOURCES = ["zgr_dropout.cu", "zgr_host.cu", "zgr_kernels.cu", "zgr_linear.cu", "zgr_noalloc.cu", "zgr_staged.cu", "zgr_subspace.cu", "zgr_tile.cu", "zgr_umma.cu"]
BIND_SOURCE = "zgr_bind.cpp"


def bind_path() -> str:
    """The marshalling module of this torch and this Python.  Their versions are in its name: it is compiled against torch's C++ headers, and
    one that was built for another torch would misread its tensors without a word."""
    return os.path.join(_HERE, f"_zgr_bind-{importlib.metadata.version('torch')}-{sys.implementation.cache_tag}.so")


def _newest(paths) -> float:
    return max(os.path.getmtime(p) for p in paths)


def _current(out: str, sources) -> bool:
    return os.path.exists(out) and os.path.getmtime(out) >= _newest(sources)


def build(force: bool = False, verbose: bool = False) -> str:
    header = os.path.join(_ROOT, "include", "zgr.h")
    sources = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != BIND_SOURCE] + [header]
    if force or not _current(LIB, sources):
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        tmp = LIB + f".tmp{os.getpid()}"
        cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared",
               "-Xcompiler", "-fPIC", "-I", os.path.join(_ROOT, "include"), "-I", CSRC, "-o", tmp]
        if verbose:
            cmd += ["-Xptxas", "-v"]
        cmd += [os.path.join(CSRC, s) for s in SOURCES]
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    if force or not _current(bind_path(), [os.path.join(CSRC, BIND_SOURCE), header]):
        _build_bind()
    return LIB


def _build_bind() -> None:
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    bind = bind_path()
    tmp = bind + f".tmp{os.getpid()}"
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=1",
                    "-isystem", os.path.join(torch, "include"), "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                    "-isystem", os.path.join(cuda, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(_ROOT, "include"),
                    os.path.join(CSRC, BIND_SOURCE), "-o", tmp, "-L", os.path.join(torch, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"],
                   check=True)
    os.replace(tmp, bind)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
