"""Compile the hch shared library for gfx950 with hipcc (in-tree, next to the sources)."""
from __future__ import annotations

import hashlib
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhch.so")
SOURCES = ["hch_api.hip", "psh_build.cpp", "norm_rope.hip", "attn_bf16.hip", "attn_f32.hip", "attn_api.hip"]
# accumulators of the matrix instructions in ordinary VGPRs, updated in place: with
# the default (AGPR) form the compiler copies every accumulator through VGPRs once per loop
# iteration, which costs the bf16 kernels more issue slots than their matrix instructions
VGPR_FORM = ("hch_api.hip", "attn_bf16.hip", "attn_f32.hip")
HEADERS = ["kernels.hip.hpp", "direct.hip.hpp", "gemm_bf16.hip.hpp", "split_wgrad.hip.hpp", "split_conv.hip.hpp", "conv_small.hip.hpp", "split_columns.hip.hpp", "split_dcol.hip.hpp", "split_field.hip.hpp", "conv_bf16.hip.hpp", "psh_device.hip.hpp", "occupancy.hip.hpp", "psh_build.hpp", "profile.hpp", "api_common.hpp", "norm.hip.hpp", "rope.hip.hpp", "attn.hip.hpp", "attn_launch.hpp", os.path.join("..", "..", "include", "hch.h")]


def hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def source_digest():
    """First 16 hex digits of a sha256 over the library's sources (csrc/ and the public header):
    names the code a measurement was taken on (the summaries under profiles/ carry it, bench.py
    compares it with the sources it runs)."""
    h = hashlib.sha256()
    paths = [os.path.join(CSRC, n) for n in sorted(os.listdir(CSRC))]
    paths.append(os.path.join(HERE, "..", "include", "hch.h"))
    for p in paths:
        with open(p, "rb") as f:
            h.update(os.path.basename(p).encode())
            h.update(f.read())
    return h.hexdigest()[:16]


def build_library(force=True, verbose=False):
    """Build libhch.so.  With force=False an up-to-date library is kept."""
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    if not force and os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in deps):
        return LIB
    base = [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
            # keep the compiler from forming packed-fp32 instructions
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-pthread"] + os.environ.get("HCH_EXTRA_HIPCC_FLAGS", "").split()

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        subprocess.check_call(cmd)

    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, f + ".o") for f in SOURCES]
        with ThreadPoolExecutor(max_workers=len(SOURCES)) as pool:
            list(pool.map(run, [base + (["-mllvm", "-amdgpu-mfma-vgpr-form"] if f in VGPR_FORM else [])
                                + ["-c", os.path.join(CSRC, f), "-o", o] for f, o in zip(SOURCES, objects)]))
        run(base + ["-shared", "-o", LIB] + objects)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
