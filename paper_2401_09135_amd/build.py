"""Builds libals.so (HIP, gfx950) in-tree: one object per source compiled in parallel, then
one shared library next to this file."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libals.so")
SOURCES = ["host.cpp", "elementwise.hip", "gemm_generic.hip", "gemm_mfma_f32.hip", "gemm_mfma_any.hip", "gemm_mfma_deep.hip", "gemm_mfma.hip",
           "fp8_quant.hip", "norm_fp8.hip", "gemm_fp8.hip", "gemm_fp8_e4m3_e4m3.hip", "gemm_fp8_e4m3_e5m2.hip",
           "gemm_fp8_e5m2_e4m3.hip", "gemm_fp8_e5m2_e5m2.hip", "grad_norm.hip",
           "attention_generic.hip", "attention_mfma_f32.hip", "attention_mfma_any.hip", "attention_mfma.hip", "context.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = ["hipcc", "-x", "hip", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
