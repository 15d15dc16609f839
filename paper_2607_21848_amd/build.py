"""Build librevisit.so in-tree with hipcc for gfx950.

Usage: ``python -m paper_2607_21848_amd.build`` (or ``build()`` from Python).
The shared library lands next to this file; the Python binding loads it
from there.
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "librevisit.so")
SOURCES = ["capi.cpp", "retrieve.hip", "reproject.hip", "attention.hip", "kvpack.hip", "stream.cpp", "stream_kernels.hip",
           "rotary.hip", "keyweight.hip", "select.hip", "compact.hip", "paged_append.hip"]
# compiled with the matrix instructions accumulating in the registers that vector instructions read: a kernel of more
# than 256 registers otherwise gets the others, and a move for each element that it reads
WIDE_SOURCES = ["paged_attention.hip", "paged_tile.hip"]
WIDE_FLAGS = ["-mllvm", "-amdgpu-mfma-vgpr-form"]
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (set HIPCC or install ROCm)")


def compile_flags():
    return [
        f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
        "-Wall", "-Wno-unused-function",
        # packed fp32 instructions are kept out of every kernel
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-I", os.path.join(os.path.dirname(PKG_DIR), "include"),
    ]


def build(verbose: bool = False) -> str:
    """Compile every source and link librevisit.so; returns its path."""
    cc = hipcc()
    objdir = os.path.join(PKG_DIR, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    for src in SOURCES + WIDE_SOURCES:
        obj = os.path.join(objdir, src.rsplit(".", 1)[0] + ".o")
        lang = ["-x", "hip"] if src.endswith(".hip") else []
        cmd = [cc, *compile_flags(), *(WIDE_FLAGS if src in WIDE_SOURCES else []), *lang, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        objs.append(obj)
    tmp = LIB_PATH + ".tmp"
    cmd = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
