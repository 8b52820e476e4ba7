"""Build the gfx950 HIP library libroi_extract.so in-tree (hipcc, no JIT cache).

Flags:
  --offload-arch=gfx950          MI355X (CDNA4) only
  -ffp-contract=off              sample geometry is one rounding per written operation
  -munsafe-fp-atomics            fp32 atomicAdd becomes the hardware global_atomic_add_f32
  -target-feature -packed-fp32-ops   no packed fp32 arithmetic in generated code
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIBRARY = os.path.join(HERE, "libroi_extract.so")
SOURCES = ["api.hip", "plan.hip", "fwd.hip", "bwd.hip", "adaptive.hip", "pool.hip", "deform.hip", "nms.hip", "select.hip",
           "relation_api.hip", "attn_dense.hip", "attn_recall.hip", "attn_bwd.hip", "memory.hip", "norm.hip",
           "head_api.hip", "gemm_bf16.hip", "gemm_f32.hip", "linear.hip", "logprob.hip", "evict_api.hip", "weigh.hip",
           "evict.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-munsafe-fp-atomics", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-I", INCLUDE, "-I", CSRC]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    subprocess.check_call([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library (always rebuilds)."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIBRARY + ".tmp%d" % os.getpid()
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    os.replace(tmp, LIBRARY)
    if verbose:
        print("built", LIBRARY)
    return LIBRARY


if __name__ == "__main__":
    build(verbose=True)
