"""Build the gfx950 libraries ``libdtree.so`` and ``libdscores.so`` in-tree with hipcc.

    python -m paper_1111_1373_amd.build

All HIP code is compiled with packed-FP32 instruction selection disabled, IEEE f32
denormals kept (no flush to zero) and no floating-point contraction or fast-math, so the
threshold comparisons keep exact IEEE semantics.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libdtree.so")
OBJDIR = os.path.join(HERE, "_build")
SOURCES = ["dtree.hip", "kernels.hip", "kernels_f16.hip", "kernels_bf16.hip", "kernels_u8.hip",
           "forest.hip", "forest_ex16.hip",
           "forest_packed.hip", "forest_list.hip", "forest_spec.hip", "probe.hip", "path.hip", "encode.cpp", "pipeline.cpp"]
# operators on rows of class scores: a library of their own, which needs no tree
SCORES_LIB = os.path.join(HERE, "libdscores.so")
SCORES_SOURCES = ["scores.cpp", "scores_top.hip", "scores_sample.hip", "scores_distill.hip"]
ARCH = "gfx950"

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=" + ARCH,
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fno-gpu-flush-denormals-to-zero", "-ffp-contract=off", "-fno-fast-math",
    "-Wall", "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    return "hipcc"


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    cmd = [hipcc()] + HIPCC_FLAGS + ["-x", "hip", "-I", INCLUDE, "-I", CSRC, "-c", "-o", obj, src]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return obj


def _link(lib: str, objs, verbose: bool) -> None:
    tmp = lib + ".tmp%d" % os.getpid()
    cmd = [hipcc(), "-shared", "-fPIC", "--hip-link", "--offload-arch=" + ARCH, "-o", tmp] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    """Compile every translation unit (in parallel) and link the libraries; returns libdtree.so."""
    from concurrent.futures import ThreadPoolExecutor

    os.makedirs(OBJDIR, exist_ok=True)
    srcs = [os.path.join(CSRC, s) for s in SOURCES + SCORES_SOURCES]
    jobs = max(1, min(len(srcs), os.cpu_count() or 1))
    with ThreadPoolExecutor(jobs) as pool:
        objs = list(pool.map(lambda s: _compile(s, verbose), srcs))
    _link(LIB, objs[:len(SOURCES)], verbose)
    _link(SCORES_LIB, objs[len(SOURCES):], verbose)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIB)
