"""Build libdro.so, the gfx950 HIP library behind include/dro.h.

    python -m paper_2607_16892_amd.build

Each translation unit is compiled for gfx950 with packed-FP32 instructions
disabled; the exact / capacity translation units also disable FMA
contraction so every double expression is rounded exactly as written.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdro.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

COMMON = ["-O3", "-fPIC", "-std=c++17", f"--offload-arch={ARCH}",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-I", INCLUDE, "-I", CSRC, "-Wall", "-Wno-unused-result"]
UNITS = {
    "dense.hip": ["-ffp-contract=off"],
    "exact.hip": ["-ffp-contract=off"],
    "serving.hip": ["-ffp-contract=off"],
    "api.hip": ["-ffp-contract=off"],
    "kv_api.hip": [],
    "kv_cache.hip": ["-ffp-contract=off"],
    "kv_attention.hip": [],
    "kv_decode_bf16.hip": [],
    "kv_decode_f16.hip": [],
    "kv_prefill_bf16.hip": [],
    "kv_prefill_f16.hip": [],
}


def _compile(unit: str, extra: list[str]) -> str:
    obj = os.path.join(BUILD, unit.replace(".hip", ".o"))
    cmd = [HIPCC, "-c", os.path.join(CSRC, unit), "-o", obj] + COMMON + extra
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {unit}:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(UNITS)) as ex:
        objs = list(ex.map(lambda kv: _compile(*kv), UNITS.items()))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
