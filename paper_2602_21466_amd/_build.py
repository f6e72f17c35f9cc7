"""Compiles the HIP library (libcgtp.so: full CGTP and the MIMO signal products) in-tree for gfx950 with hipcc."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libcgtp.so")
SOURCES = [os.path.join(HERE, "csrc", f) for f in
           ("cgtp_plan.cpp", "cgtp_kernels.hip", "cgtp_kernels_channels.hip", "cgtp_backward.hip", "cgtp_direct.hip", "cgtp_direct_backward.hip", "cgtp_kernels_real.hip", "istp_plan.cpp", "istp_kernels.hip", "istp_kernels_real.hip",
            "istp_kernels_channels.hip", "istp_kernels_tensor.hip", "istp_kernels_channels_tensor.hip",
            "istp_real.hip", "ffn_plan.cpp", "ffn_gemm.hip",
            "ffn_tile_bf16.hip", "ffn_tile_fp16.hip", "ffn_tile_fp32.hip", "ffn_few_bf16.hip", "ffn_few_fp16.hip", "ffn_few_fp32.hip", "ffn_few_grad.hip",
            "ffn_norm_bf16.hip", "ffn_norm_fp16.hip", "ffn_norm_fp32.hip",
            "ffn_layer.cpp", "ffn_layer_bf16.hip", "ffn_layer_fp16.hip", "ffn_layer_fp32.hip",
            "experts_plan.cpp", "ffn_route.hip", "ffn_experts_bf16.hip", "ffn_experts_fp16.hip", "ffn_experts_fp32.hip",
            "ffn_experts_few_bf16.hip", "ffn_experts_few_fp16.hip", "ffn_experts_few_fp32.hip")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# Packed FP32 instructions are switched off for all device code.
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-Wall", "-Wno-unused-result"]


def build(force: bool = True, extra=None) -> str:
    """Compiles every source to an object, as many at a time as there are processors, then links the library."""
    if not force and os.path.exists(LIB):
        return LIB
    tag = ".tmp%d" % os.getpid()
    objs = [os.path.join(HERE, "csrc", os.path.basename(src) + tag + ".o") for src in SOURCES]
    compile_flags = [f for f in FLAGS if f != "-shared"]
    compile_one = lambda src, obj: subprocess.run([HIPCC] + compile_flags + list(extra or []) + ["-c", src, "-o", obj]).returncode
    with concurrent.futures.ThreadPoolExecutor(min(os.cpu_count() or 1, 16)) as pool:
        failed = [src for src, rc in zip(SOURCES, pool.map(compile_one, SOURCES, objs)) if rc != 0]
    try:
        if failed:
            raise subprocess.CalledProcessError(1, "hipcc", "failed: %s" % ", ".join(failed))
        tmp = LIB + tag
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", tmp], check=True)
        os.replace(tmp, LIB)
    finally:
        for obj in objs:
            if os.path.exists(obj):
                os.remove(obj)
    return LIB


if __name__ == "__main__":
    print(build())
