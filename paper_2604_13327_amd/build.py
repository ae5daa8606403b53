"""Builds libetc.so (the HIP megakernel + C ABI) in-tree for gfx950."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libetc.so")
SOURCES = ["api.cpp", "graph.cpp", "megakernel.hip", "serving.cpp", "serving.hip", "chunk_attn.hip"]
HEADERS = ["etc_types.h", "arm_args.h", "graph.h", "device_rt.hip.h", "task_gemm.hip.h", "task_attn.hip.h", "task_moe.hip.h",
           "serving.h", "serving_rt.hip.h"]


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(HERE, "..", "include", "etc.h")]
    return any(os.path.exists(d) and os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    """hipcc cross-compiles for gfx950 without a GPU."""
    if not force and not needs_build():
        return LIB
    cmd = ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-shared", "-fPIC",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-command-line-argument",
           "-o", LIB] + [os.path.join(CSRC, f) for f in SOURCES]
    if verbose:
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(True, True))
