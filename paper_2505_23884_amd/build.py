"""Builds liblact.so (the gfx950 HIP kernels + the C ABI) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "liblact.so")
SOURCES = ["lact_api.hip", "lact_kernels.hip", "lact_io.hip", "lact_attn_api.hip", "lact_window.hip", "lact_paged.hip",
           "lact_rope.hip", "lact_codes.hip", "lact_prefix.hip", "lact_prefix_bf16.hip",
           "lact_prefix_e4m3.hip", "lact_prefix_e4m3_fp32.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU ops stay off: plain fp32 math only
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = False) -> str:
    """Compile every HIP source (side by side) and link liblact.so next to this file; returns its path."""
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as objs, ThreadPoolExecutor(max_workers=8) as pool:
        def run(cmd):
            if verbose:
                print(" ".join(cmd), flush=True)
            res = subprocess.run(cmd, capture_output=True, text=True)
            if res.returncode != 0:
                sys.stderr.write(res.stdout + res.stderr)
                raise RuntimeError(f"hipcc failed ({res.returncode}) building {LIB}")

        def compile_one(src):
            obj = os.path.join(objs, src + ".o")
            run([hipcc(), *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, src),
                 "-o", obj])
            return obj

        objects = list(pool.map(compile_one, SOURCES))
        run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
