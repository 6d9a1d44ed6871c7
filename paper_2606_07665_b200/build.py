"""Builds libac.so (the C-ABI library) in-tree with nvcc for sm_100a.

    python -m paper_2606_07665_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libac.so")
SOURCES = ["ac_api.cu", "rope_kv_append.cu", "paged_decode_attn.cu", "splitkv_merge.cu",
           "attn_static_scratch.cu", "qkv_prelude.cu", "stage_inputs.cu", "proj_tc.cu", "hbm_probe.cu",
           "q4_attn.cu", "q4_cache.cu", "cache_pages.cu"]
HEADERS = [os.path.join(CSRC, "ac_device.cuh"), os.path.join(CSRC, "ac_internal.h"),
           os.path.join(CSRC, "rope_variant.cuh"), os.path.join(CSRC, "split_merge.cuh"),
           os.path.join(CSRC, "q4_format.cuh"),
           os.path.join(ROOT, "include", "ac.h")]


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def up_to_date() -> bool:
    if not os.path.exists(LIB_PATH):
        return False
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return all(os.path.getmtime(d) <= t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB_PATH
    cmd = [nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-diag-suppress", "550",
           "-shared", "-Xcompiler", "-fPIC", "-cudart", "static", "--threads", "0",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", LIB_PATH]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed building libac.so")
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
