"""Build librsa.so (HIP, gfx950 only) in-tree with hipcc.

Usage: ``python -m paper_2511_19835_amd.build`` or ``build_library()``.
The shared object lands next to this file so it travels with the source tree.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(HERE, "librsa.so")

SOURCES = [
    "rsa_api.hip",
    "pool_kernels.hip",
    "score_kernels.hip",
    "gapr_kernels.hip",
    "select_kernels.hip",
    "adjacency_kernels.hip",
    "reorder_kernels.hip",
    "attn_side_kernels.hip",
    "attn_kernels.hip",
    "cache_api.hip",
    "cache_page_kernels.hip",
    "cache_select_kernels.hip",
    "cache_attn_kernels.hip",
    "serve_api.hip",
    "assign_kernels.hip",
    "rotary_kernels.hip",
    "fourbit_page_kernels.hip",
    "fourbit_attn_kernels.hip",
]

# Packed-fp32 VALU forms (v_pk_*_f32) are switched off for every device translation unit.
HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: librsa.so cannot be built")
    return exe


def _compile(src: str, obj: str, extra) -> None:
    cmd = [_hipcc(), *HIP_FLAGS, *extra, "-I", INCLUDE, "-I", CSRC, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{out}")
    if out.strip():
        sys.stderr.write(out + "\n")


def build_library(extra_flags=(), jobs: int = 6, verbose: bool = True) -> str:
    build_dir = os.path.join(HERE, "_build")
    os.makedirs(build_dir, exist_ok=True)
    objs = [os.path.join(build_dir, s.replace(".hip", ".o")) for s in SOURCES]
    with concurrent.futures.ThreadPoolExecutor(max_workers=jobs) as ex:
        futs = [ex.submit(_compile, s, o, list(extra_flags)) for s, o in zip(SOURCES, objs)]
        for f in futs:
            f.result()
    tmp = LIB_PATH + ".tmp"
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB_PATH)
    if verbose:
        print(f"built {LIB_PATH}")
    return LIB_PATH


if __name__ == "__main__":
    build_library()
