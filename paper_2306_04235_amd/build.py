"""Build libmnmt.so (HIP kernels for gfx950 + host code) in-tree with hipcc.

Floating point is compiled for reproducible IEEE binary32: no contraction
(every fma is written out), denormals kept, correctly rounded division and
square root, and the packed-fp32 instructions disabled.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmnmt.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

COMMON = ["-O3", "-fPIC", "-std=c++17", "-ffp-contract=off", "-Wall", "-Wno-unused-function",
          "-I" + os.path.join(os.path.dirname(HERE), "include")]
DEVICE = [f"--offload-arch={ARCH}", "-fno-gpu-flush-denormals-to-zero", "-fhip-fp32-correctly-rounded-divide-sqrt",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# per-file device flags: matrix-core accumulators in VGPRs
EXTRA = {f: ["-mllvm", "-amdgpu-mfma-vgpr-form"] for f in ("gemm.hip", "attn_paged.hip", "attn_cross.hip")}
SOURCES = ["qlinear.hip", "kernels.hip", "decode_fused.hip", "decode_step.hip", "decode_rows.hip", "encode_rows.hip", "encode_small.hip", "gemm.hip", "logits.hip",
           "noalloc.hip", "pages.hip", "attn_paged.hip", "attn_cross.hip", "model.cpp", "session.cpp", "api.cpp", "cache.cpp"]


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, src + ".o")
    path = os.path.join(CSRC, src)
    flags = COMMON + (DEVICE + EXTRA.get(src, []) if src.endswith(".hip") else ["-D__HIP_PLATFORM_AMD__"])
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [HIPCC, *flags, *lang, "-c", path, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n{r.stdout}\n{r.stderr}")
    warn = [ln for ln in r.stderr.splitlines() if "packed-fp32-ops" not in ln and ln.strip()]
    if warn and verbose:
        print("\n".join(warn))
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", LIB + ".tmp", *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
