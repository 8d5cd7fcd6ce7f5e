"""Build libsrq.so (the C-ABI library) from the HIP sources with hipcc, for gfx950 only.

Flags that matter:
  -ffp-contract=off            every binary32 step of the quantizer rounds once (no fma fusion)
  -target-feature -packed-fp32-ops   no packed-fp32 VALU forms
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsrq.so")
SOURCES = ["srq_quantize.hip", "srq_quantize_jobs.hip", "srq_quantize_dual.hip", "srq_gemm.hip", "srq_fused.hip", "srq_update.hip", "srq_api.hip",
           "srq_blocks.hip", "srq_norm.hip", "srq_gated.hip", "srq_block_gemm.hip", "srq_blocks_api.hip",
           "srq_attention.hip", "srq_attention_bwd.hip", "srq_embedding.hip", "srq_adamw.hip", "srq_decoder_api.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function",
         "-Wno-unknown-attributes"]


def _compile(src):
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    subprocess.run([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj], check=True)
    return obj


def build(verbose=False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs], check=True)
    if verbose:
        print("built", LIB)
    return LIB


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "srq.h")]
    return any(os.path.getmtime(d) > t for d in deps)


if __name__ == "__main__":
    build(verbose=True)
