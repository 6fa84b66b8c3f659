"""Builds libslowmo.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libslowmo.so")
SOURCES = ["slowmo_kernels.hip", "slowmo_heads.hip", "slowmo_orth.hip", "slowmo_orth.cpp", "slowmo_api.cpp", "slowmo_plan.cpp",
           "slowmo_attention.hip", "slowmo_attention_backward.hip", "slowmo_append.hip"]
HEADERS = ["slowmo_kernels.h", "slowmo_plan.h", "slowmo_status.h", "slowmo_orth.h", "slowmo_attention.h",
           os.path.join("..", "..", "include", "slowmo.h"),
           os.path.join("..", "..", "include", "slowmo_operators.h"),
           os.path.join("..", "..", "include", "slowmo_attention.h")]

# -ffp-contract=off: every product and sum rounds on its own, in source order
# (the order of the paper's formulas); the packed-fp32 feature is disabled.
# Kernel-argument preload: the first 14 words of a kernel's arguments are in its scalar registers when a
# wave starts, one trip to memory less in front of its first load (short lists: a step of 4.9 us 0.2-0.3
# us less, 0.95-0.97 of a round; long lists 0.99-1.00).  The words that lead to a wave's data come first.
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wextra",
         "-Wno-unused-parameter", "-mllvm", "-amdgpu-kernarg-preload-count=14"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + r.stderr)
        return r.stderr

    # Every source by itself, side by side: 70 s for 180 s of processor time (8 cores).
    with tempfile.TemporaryDirectory() as made, ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = [os.path.join(made, s + ".o") for s in SOURCES]
        compile_flags = [f for f in FLAGS if f != "-shared"]
        said = list(pool.map(run, [[hipcc(), *compile_flags, "-x", "hip", "-c", os.path.join(CSRC, s), "-o", o]
                                   for s, o in zip(SOURCES, objects)]))
        said.append(run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", LIB]))
    # the host pass does not know the device-only target feature; that warning is expected
    err = "\n".join(ln for ln in "".join(said).splitlines() if "packed-fp32-ops" not in ln)
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
