"""Build ``liblazyattn.so`` in-tree for gfx950 with hipcc (cross-compiles without a GPU).

Usage: ``python -m paper_2606_04302_amd.build`` or ``paper_2606_04302_amd.build.build()``.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "liblazyattn.so")
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", shutil.which("hipcc") or "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", shutil.which("g++") or "g++")

# Packed fp32 VALU ops are disabled for every HIP translation unit: some of their forms have produced silently
# wrong results on this hardware, so the compiler must not form them from scalar or float2 code.
HIP_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC, "-Wall", "-fvisibility=hidden",
]
HOST_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", INCLUDE, "-Wall", "-Wextra"]

SOURCES = [
    ("lazy_attn_kernels.hip", "hip"),
    ("lazy_attn_api.cpp", "hip"),
    ("lazy_attn_validate.cpp", "host"),
    ("lazy_attn_plan.cpp", "host"),
    ("lazy_attn_pool.cpp", "host"),
    ("lazy_attn_backward.hip", "hip"),
    ("lazy_attn_backward_api.cpp", "hip"),
    ("lazy_attn_backward_plan.cpp", "host"),
    ("lazy_attn_evict.hip", "hip"),
    ("lazy_attn_evict_api.cpp", "hip"),
]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    # hipcc's host pass does not know the packed-fp32 target feature and says so; that line is noise.
    err = "\n".join(ln for ln in res.stderr.splitlines() if "is not a recognized feature" not in ln)
    if res.returncode != 0:
        raise RuntimeError(f"build step failed ({res.returncode}): {' '.join(cmd)}\n{res.stdout}\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library; always rebuilds.  Returns the library path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    jobs = []
    for src, kind in SOURCES:
        obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
        path = os.path.join(CSRC, src)
        if kind == "hip":
            cmd = [HIPCC, *HIP_FLAGS, "-c", path, "-o", obj]
        else:
            cmd = [CXX, *HOST_FLAGS, "-c", path, "-o", obj]
        jobs.append((cmd, obj))
    with cf.ThreadPoolExecutor(max_workers=len(jobs)) as ex:
        list(ex.map(lambda j: _run(j[0], verbose), jobs))
    tmp = LIB_PATH + ".tmp"
    _run([HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *[o for _, o in jobs]], verbose)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
