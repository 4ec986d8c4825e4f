"""Builds libivf.so (the gfx950 HIP library behind include/ivf.h) with hipcc.

Every source is compiled for gfx950 only, with floating-point contraction off
(the fp64 re-evaluation must be the exact operation sequence of the
definition: one subtraction and one fma per dimension) and packed-FP32 code
generation disabled.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libivf.so")

SOURCES = ["api.cpp", "screen.hip", "screen_i8.hip", "screen_f16.hip", "select.hip", "fallback.hip", "resolve.hip", "lists.hip", "lists_radix.hip", "kmeans.hip", "layout.hip", "pq.hip", "assign_graph.hip", "adc.hip", "probe.hip",
           "api_kv.cpp", "kv_plan.hip", "kv_pages.hip", "kv_cache.hip", "kv_select.hip", "kv_attend.hip", "kv_attend_terms.hip", "kv_prompt.hip",
           "kv_prompt_terms.hip", "api_sample.cpp", "sample.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17",
    "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]

# The PQ screen takes maxima of values whose low bits are integers; quieting
# NaNs there would cost an instruction per value (inputs are finite).
#
# The attention kernels rescale their accumulators with vector instructions
# now and then; held in the accumulation registers they would be moved there
# and back on every step (64 moves of 500 instructions at 128 channels).
VGPR_MFMA = ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]
EXTRA_FLAGS = {"pq.hip": ["-fno-honor-nans"], "kv_attend.hip": VGPR_MFMA, "kv_attend_terms.hip": VGPR_MFMA,
               "kv_prompt.hip": VGPR_MFMA, "kv_prompt_terms.hip": VGPR_MFMA}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *EXTRA_FLAGS.get(src, []), "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), r.stderr))
    return obj


def build(verbose: bool = False) -> str:
    """Compiles every source (always) and links libivf.so in the package dir."""
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
