"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache involved)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libmq.so")
SOURCES = ["mq_api.cu", "mq_fwht_quant.cu", "mq_pack.cu", "mq_aifs.cu", "mq_gemm.cu", "mq_noalloc.cu", "mq_rms.cu", "mq_gemv.cu", "mq_dynquant.cu", "mq_probe.cu", "mq_kron.cu", "mq_glue.cu", "mq_attn.cu", "mq_kv_append.cu",
           "mq_kv_attn.cu", "mq_kv_chunk.cu", "mq_kv_weights.cu", "mq_kv_weights_chunk.cu", "mq_kv_evict.cu", "mq_sample.cu", "mq_kv_plan.cu",
           "mq_kv_shared.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "mq.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into paper_2502_00425_b200/libmq.so; returns its path."""
    if not force and not _stale():
        return LIB_PATH
    cmd = [_nvcc(), "-t", "0", "-shared", "-Xcompiler", "-fPIC", "-std=c++17", "-O3", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", LIB_PATH]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
