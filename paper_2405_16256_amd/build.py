"""Builds libhh.so (the C-ABI library of hand-written gfx950 kernels) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libhh.so")
SOURCES = ["hh_api.cpp", "predictor.cpp", "elementwise.hip", "gemm_f32.hip", "gemm_f32_long_k.hip", "gemm_bf16.hip", "attn_f32.hip", "attn_bf16.hip", "scratch.hip",
           "hh_train.cpp", "head.hip", "tensors.hip"]
# Packed fp32 instructions are kept out of the generated code on purpose.  Up to 14 words of a kernel's arguments, as far as the first
# struct among them, arrive in registers instead of being loaded by every workgroup: the attention kernels' pointers, 3 or 4 words
# of the GEMMs on rings, none of the 256x256 ones.  Steps of hidden 256, 128 tokens: fp32 78.9 -> 77.3 us, 4 bf16 layers of 8
# micro-batches 395 -> 390; of hidden 1024, 700 tokens, bf16 179 -> 178; GEMMs alone and large layers take the same.
FLAGS = ["--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm", "-amdgpu-kernarg-preload-count=14",
         "-Wno-unused-command-line-argument"]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc(), *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, r.stderr[-4000:]))
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    r = subprocess.run([_hipcc(), "-shared", "-fPIC", "-o", LIB, *objs], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr[-4000:])
    if verbose:
        print("built", LIB, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
