"""Build step: compiles the C-ABI library (host tile-map builder + gfx950 HIP kernels) in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libblindsight.so")
SOURCES = ["tilemap.cpp", "device_map.hip", "attn_prefill.hip", "attn_rows.hip", "attn_f32.hip", "characterize.hip", "rope.hip", "attn_decode.hip", "cache_evict.hip"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def command(out: str = LIB, extra=()):
    return [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
            "-falign-loops=64",   # the step loops of the attention kernels: d = 64 prompt of 9K tokens 972 -> 963 us a pass
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-command-line-argument",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC, *extra, *os.environ.get("BS_EXTRA_HIPCC_FLAGS", "").split(),
            "-o", out, *[os.path.join(CSRC, s) for s in SOURCES]]


def build(verbose: bool = True) -> str:
    cmd = command()
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "blindsight.h")]
    return any(os.path.getmtime(d) > t for d in deps)


if __name__ == "__main__":
    build()
    sys.exit(0)
