"""Build libmetro.so (HIP for gfx950) in-tree.

    python -m paper_2411_03519_amd.build          # or: python paper_2411_03519_amd/build.py

Every source is compiled with hipcc for gfx950 only (objects under
``_build/``), then linked into ``paper_2411_03519_amd/libmetro.so``.  Packed
fp32 instructions are disabled for all device code.
"""

from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libmetro.so")
BUILD = os.path.join(ROOT, "_build")

SOURCES = [
    "csrc/kv_pool.cpp",
    "csrc/scheduler.cpp",
    "csrc/engine.cpp",
    "csrc/runtime.hip",
    "csrc/kernels/elementwise.hip",
    "csrc/kernels/gemm.hip",
    "csrc/kernels/attention.hip",
    "csrc/ops_fp8.hip",
    "csrc/kernels/rows_fp8.hip",
    "csrc/kernels/route.hip",
    "csrc/kernels/gemm_fp8.hip",
    "csrc/ops_draft.hip",
    "csrc/kernels/append.hip",
    "csrc/kernels/attn_tree.hip",
    "csrc/kernels/sample.hip",
]

ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", shutil.which("hipcc") or "/opt/rocm/bin/hipcc")
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-result", f"-I{ROOT}/include"]
DEVICE = [f"--offload-arch={ARCH}", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src: str) -> str:
    path = os.path.join(PKG, src)
    obj = os.path.join(BUILD, src.replace("/", "_") + ".o")
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [HIPCC, *COMMON, *DEVICE, *lang, "-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print("built", OUT)
    return OUT


if __name__ == "__main__":
    try:
        build()
    except RuntimeError as e:
        print(e, file=sys.stderr)
        sys.exit(1)
