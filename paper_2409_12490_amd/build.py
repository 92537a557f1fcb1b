"""Compile the HIP sources under csrc/ into paper_2409_12490_amd/libcritiprefill.so (gfx950 only)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libcritiprefill.so")
SOURCES = ["api.hip", "estimate.hip", "select.hip", "attn_fp32.hip", "attn_fp32_split.hip", "attn_bf16.hip", "attn_bf16_rows.hip", "attn_bf16_half.hip",
           "cache_api.hip", "norm_rope.hip", "attn_paged.hip", "attn_paged_chunk.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# bf16 attention: MFMA results stay in architectural VGPRs (S^T feeds the softmax VALU code directly; the
# operands that only MFMA touches live in AGPRs), and fmaxf needs no NaN-quieting pre-pass (the kernel
# never produces NaN: masked logits are -inf and the running max is guarded).  attn_paged.hip takes the former
# alone: 32 fp32 rows lose 64 copies a step (20 x 200 tokens after 8000, 4/2 heads, 724 -> 684 us), 64 rows their
# spills (1 x 16 tokens after 3000, 64/1 heads, 55 -> 45 us).
_BF16_ATTN = ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-fno-honor-nans", "-mno-amdgpu-ieee"]
EXTRA = {"attn_bf16.hip": _BF16_ATTN, "attn_bf16_rows.hip": _BF16_ATTN, "attn_bf16_half.hip": _BF16_ATTN,
         "attn_paged_chunk.hip": _BF16_ATTN, "attn_paged.hip": _BF16_ATTN[:2]}


def _compile(src: str, objdir: str) -> str:
    obj = os.path.join(objdir, src.replace(".hip", ".o"))
    cmd = [HIPCC, *FLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(f"hipcc failed on {src}")
    return obj


def build(verbose: bool = False) -> str:
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda s: _compile(s, objdir), SOURCES))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link failed")
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
