"""Builds ``libatspeed.so`` (gfx950, hipcc) and ``_marshal.so`` (its calls on PyTorch tensors, g++) in this directory.

``python -m paper_2410_05165_amd.build library`` builds the first alone.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libatspeed.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = ["runtime.hip", "gemm.hip", "gemm_f32.hip", "attention.hip", "misc.hip", "select.hip", "relaxed.hip", "align.hip",
           "paged.hip", "tree_attention.hip", "rules.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-result", "-fvisibility=hidden"]


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(os.path.basename(cmd[0]) + " failed")


def build(verbose: bool = False) -> str:
    build_library(verbose)
    build_marshal(verbose)
    return LIB


def build_library(verbose: bool = False) -> str:
    """libatspeed.so alone, all that a caller of include/atspeed.h needs: hipcc, no PyTorch."""
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        list(pool.map(lambda so: _run([HIPCC, *FLAGS, "-c", os.path.join(CSRC, so[0]), "-o", so[1]], verbose),
                      zip(SOURCES, objects)))
        _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB + ".tmp"], verbose)
    os.replace(LIB + ".tmp", LIB)
    return LIB


def build_marshal(verbose: bool = False) -> str:
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths

    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *["-I" + p for p in (*include_paths(), sysconfig.get_paths()["include"])],
           os.path.join(CSRC, "marshal.cpp"), "-o", MARSHAL + ".tmp",
           "-L" + os.path.join(os.path.dirname(torch.__file__), "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python",
           "-L" + HERE, "-l:libatspeed.so", "-Wl,-rpath,$ORIGIN"]
    _run(cmd, verbose)
    os.replace(MARSHAL + ".tmp", MARSHAL)
    return MARSHAL


if __name__ == "__main__":
    print(build_library(verbose=True) if sys.argv[1:] == ["library"] else build(verbose=True))
