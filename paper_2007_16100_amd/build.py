"""Build libspv.so (hand-written HIP for gfx950) in-tree.

    python -m paper_2007_16100_amd.build

Each translation unit under csrc/ is compiled with hipcc for gfx950 only and
linked into paper_2007_16100_amd/libspv.so.  The flags keep IEEE semantics (no
fast-math; HIP's default correctly rounded fp32 division, which Eq. 1's
quantization relies on) and disable packed-fp32 instruction selection.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libspv.so")
BUILD_DIR = os.path.join(HERE, "_build")
SOURCES = ["hash_sort_scan.hip", "radix.hip", "voxelize.hip", "kmap.hip", "conv.hip", "conv_union.hip", "conv_up.hip", "devox.hip",
           "linear.hip", "norm.hip", "attention.hip", "attention_backward.hip", "rope.hip", "group_norm.hip",
           "checkpoint8.hip", "backward.hip", "api.hip"]
ARCH = os.environ.get("SPV_OFFLOAD_ARCH", "gfx950")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

CFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
    "-fno-fast-math", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *CFLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 4)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print("built", OUT)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
