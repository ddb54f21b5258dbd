"""Builds csrc/libdifr.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(CSRC, "libdifr.so")
SOURCES = ["difr_api.cu", "difr_mx_api.cu", "k0_expand_seeds.cu", "k1_fused_score.cu", "k2_finalize.cu",
           "k2_filtered.cu", "k2_select.cu", "k3_detect.cu", "k4_norm.cu", "k5_mx_convert.cu", "k6_mx_logits.cu",
           "difr_step_api.cu", "k7_block_norm.cu", "k8_w4_convert.cu", "k9_w4_logits.cu",
           "k10_verify.cu"]
HEADERS = ["difr_device.cuh", "difr_host.h", "difr_kernels.h", "difr_plan.h", "mx_device.cuh", "mx_kernels.h",
           "norm_device.cuh", "logit_plan.h", "logit_tiles.cuh", "step_kernels.h", "w4_device.cuh",
           os.path.join("..", "..", "include", "difr.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC", "--threads", "0"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        nvcc = os.environ.get("NVCC", "nvcc")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + SOURCES + ["-lcudart"]
        subprocess.check_call(cmd, cwd=CSRC)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
