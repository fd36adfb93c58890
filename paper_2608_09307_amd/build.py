"""Build the LinSimp HIP library (liblinsimp.so) in-tree for gfx950.

    python -m paper_2608_09307_amd.build        # or build() from Python

Every source is compiled with hipcc for gfx950 only; objects go to
``_build/`` at the repository root and the shared library to
``paper_2608_09307_amd/_lib/liblinsimp.so``.
"""

from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIBDIR = os.path.join(PKG, "_lib")
LIB = os.path.join(LIBDIR, "liblinsimp.so")

SOURCES = ["api.cpp", "fwd.hip", "prefill.hip", "bwd.hip", "decode.hip", "head.hip", "bank.hip",
           "attn.hip", "glr.hip", "mixers.cpp"]
ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "-x", "hip", f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]

# Per-source additions.  The backward's machine scheduler tracks register
# pressure with the target's own trackers: when it was added the dq/dr sweep
# spilled 60 instead of 75 registers at its 256 and ran 3-4% faster (today's
# spills 24 at d = m = 128 with it and without; elsewhere the option raised
# register counts and lowered occupancy, so it stays local).  Attention's key
# sweep at d = 128 spills no register with it instead of eight: 16 heads of
# 16384 tokens 2.27 -> 2.08 ms in one session.
SOURCE_FLAGS = {"bwd.hip": ["-mllvm", "-amdgpu-use-amdgpu-trackers"],
                "attn.hip": ["-mllvm", "-amdgpu-use-amdgpu-trackers"]}


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    errs = "\n".join(line for line in res.stderr.splitlines()
                     if "packed-fp32-ops" not in line and line.strip())
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{errs}")
    if verbose and errs:
        print(errs, flush=True)
    return obj


def build(verbose: bool = False, jobs: int | None = None) -> str:
    """Compile every source for gfx950 and link liblinsimp.so; returns its path."""
    os.makedirs(BUILD, exist_ok=True)
    os.makedirs(LIBDIR, exist_ok=True)
    jobs = jobs or min(len(SOURCES), max(1, (os.cpu_count() or 2)))
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
