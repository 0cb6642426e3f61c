"""Build libpkv.so in-tree: host code with g++, the HIP kernels with hipcc
for gfx950, linked into one shared library next to this file."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libpkv.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
# Packed-FP32 instructions are kept out of the device code on purpose.
HIP_FLAGS = ["-O3", "-std=c++17", f"--offload-arch={ARCH}", "-fPIC", "-Wall",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", f"-I{INCLUDE}", f"-I{CSRC}"]
CXX_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-Wextra", f"-I{INCLUDE}", f"-I{CSRC}"]
HOST_SRC = ("plan.cpp", "serve_plan.cpp")
# The attention kernels are built once for each head_dim.
HIP_SRC = (("restore.hip", ()), ("gather.hip", ()), ("serve.hip", ()), ("evict.hip", ()),
           *((src, (f"-DPKV_HEAD_DIM={d}",)) for src in ("attend.hip", "weigh.hip") for d in (64, 128, 256)))


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"build step failed: {' '.join(cmd[:2])} ... (exit {res.returncode})")
    return res


def build(verbose: bool = False) -> str:
    """Compile and link libpkv.so; returns its path.  Always rebuilds."""
    os.makedirs(BUILD, exist_ok=True)
    cxx = shutil.which("g++") or "g++"
    steps = [(src.replace(".cpp", ".o"), [cxx, *CXX_FLAGS, "-c", os.path.join(CSRC, src)]) for src in HOST_SRC]
    for src, flags in HIP_SRC:
        obj = src.replace(".hip", "".join("_" + f.split("=")[1] for f in flags) + ".o")
        steps.append((obj, [HIPCC, *HIP_FLAGS, *flags, "-c", os.path.join(CSRC, src)]))
    objs = [os.path.join(BUILD, obj) for obj, _ in steps]
    with ThreadPoolExecutor(min(len(steps), os.cpu_count() or 1)) as pool:
        list(pool.map(lambda s: _run([*s[1], "-o", os.path.join(BUILD, s[0])], verbose), steps))
    tmp = LIB + ".tmp"
    _run([HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
