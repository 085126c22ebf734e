"""Build the HIP library ``libflashcp.so`` in-tree for gfx950 with hipcc.

Usage: ``python -m paper_2606_08476_amd.build`` (or ``build()``).
Objects go to ``_build/`` at the repository root; the shared library is
written next to this file, where the binding loads it.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libflashcp.so")
BUILD = os.path.join(ROOT, "_build")

SOURCES = [
    "host/plan.cpp",
    "host/view.cpp",
    "host/api.cpp",
    "host/noalloc.cpp",
    "host/rope.cpp",
    "host/norm.cpp",
    "kernels/attn_fwd.hip",
    "kernels/attn_fwd_cap.hip",
    "kernels/attn_fwd_bias.hip",
    "kernels/attn_fwd_cap_bias.hip",
    "kernels/attn_fwd_window.hip",
    "kernels/attn_fwd_window_cap.hip",
    "kernels/attn_fwd_window_bias.hip",
    "kernels/attn_fwd_window_cap_bias.hip",
    "kernels/attn_bwd.hip",
    "kernels/attn_bwd_cap.hip",
    "kernels/attn_bwd_bias.hip",
    "kernels/attn_bwd_cap_bias.hip",
    "kernels/attn_bwd_window.hip",
    "kernels/attn_bwd_window_cap.hip",
    "kernels/attn_bwd_window_bias.hip",
    "kernels/attn_bwd_window_cap_bias.hip",
    "kernels/attn_bwd_dq.hip",
    "kernels/elementwise.hip",
    "kernels/rope.hip",
    "kernels/norm.hip",
]

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-fPIC",
    "-std=c++17",
    "-munsafe-fp-atomics",
    "-Wall",
    "-Wno-unused-result",
    # keep the compiler from forming packed fp32 vector ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


def _hipcc() -> str:
    for c in ("/opt/rocm/bin/hipcc", "hipcc"):
        if os.path.isabs(c) and os.path.exists(c):
            return c
    return "hipcc"


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, src.replace("/", "_") + ".o")
    path = os.path.join(CSRC, src)
    # every source is compiled as HIP: the host sources launch kernels or
    # name device symbols
    lang = ["-x", "hip"]
    cmd = [_hipcc(), *FLAGS, *lang, "-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp"
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print(f"built {OUT}")
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
