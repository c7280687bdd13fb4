"""Build librft.so (the HIP kernels + C ABI) in-tree for gfx950 with hipcc.

    python -m paper_2505_17826_amd.build_lib [--verbose]

Every source is compiled on each call (a "does it build" check as much as a
build); objects go to ``_build/`` and the shared library next to this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "librft.so")
ARCH = os.environ.get("RFT_OFFLOAD_ARCH", "gfx950")

SOURCES = ["rft_abi.hip", "k_tokens.hip", "k_adv_loss.hip", "k_gemm_mfma.hip", "k_gemm_f32.hip",
           "k_layout.hip", "k_logits.hip", "k_step.hip", "k_pref.hip", "k_router.hip", "k_adamw.hip",
           "k_ortho.hip", "k_expert.hip", "k_linear.hip",
           "k_linear_few.hip", "k_linear_f32.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CFLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-I", INCLUDE, "-I", CSRC,
          # packed fp32 arithmetic is kept off for all device code
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wall", "-Wno-unused-function", "-Wno-unused-variable"]


# Per-source flags. The GEMM epilogues take maxima over accumulators and
# cross-lane moves; without NaN semantics the compiler drops the quieting of
# each operand before every max (the hardware max still returns the non-NaN
# operand, and exp/add still propagate a NaN into the sums).
# The products of k_linear's main loop are unrolled whole (accumulators are registers): more
# than the compiler's default limit for a loop that asks for it.
SOURCE_FLAGS = {"k_gemm_mfma.hip": ["-fno-honor-nans"],
                "k_linear.hip": ["-mllvm", "-pragma-unroll-threshold=200000"]}


def _compile(src, verbose=False, extra=()):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *CFLAGS, *SOURCE_FLAGS.get(src, []), *extra, "-c", os.path.join(CSRC, src),
           "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out)
    return obj


def build(verbose: bool = False, extra=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose, extra), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    v = "--verbose" in sys.argv
    extra = ["-Rpass-analysis=kernel-resource-usage"] if "--resources" in sys.argv else []
    print(build(verbose=v or bool(extra), extra=extra))
