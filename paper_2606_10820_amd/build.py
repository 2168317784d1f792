"""Build libkforcing.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2606_10820_amd.build
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libkforcing.so")
BUILD_DIR = os.path.join(PKG, "_build")

SOURCES = ["kf_api.cpp", "kf_train_api.cpp", "kf_kernels.hip", "kf_gemm.hip", "kf_blockattn.hip",
           "kf_attnbwd.hip", "kf_norm.hip", "kf_logprobs.hip", "kf_clip.hip", "kf_heads.hip",
           "kf_dropout.hip", "kf_dropnorm.hip", "kf_policy.hip"]
HEADERS = ["kf_internal.h", "kf_lds.h", "kf_attn.h", "kf_route.h", "kf_blockattn.h", "kf_rows.h",
           "kf_train.h", "kf_norm.h", "kf_dropout.h", "kf_logprobs.h"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    "-x", "hip", f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17",
    "-Wall", "-Wno-unused-function",
    # no packed fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


# Per-source flags.  The training attention rescales its MFMA accumulators
# with VALU code inside the key loop; its inline-asm LDS reads would otherwise
# make the compiler keep the accumulators in AGPRs and copy them every tile.
SOURCE_FLAGS = {"kf_blockattn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "kf_attnbwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [HIPCC] + FLAGS + SOURCE_FLAGS.get(src, []) + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print(f"built {OUT}")
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
