"""Builds ``libzqfp.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libzqfp.so")
SOURCES = ["api.cu", "actquant.cu", "packw.cu", "w4a8_gemm.cu", "w4a8_mx_gemm.cu", "noalloc.cu", "selftest.cu", "lorc.cu",
           "fp8_block_quant.cu", "fp8_block_gemm.cu", "fp8_block_few.cu", "fp8_wgrad.cu", "fp8_block_api.cu",
           "qk_norm_rope.cu", "kv_cache.cu", "kv_attention.cu", "kv_attention_few.cu", "kv_attention_rows.cu", "kv_cache_api.cu"]
HEADERS = [os.path.join(CSRC, "zq_common.cuh"), os.path.join(CSRC, "w4a8_gemm_shared.cuh"), os.path.join(CSRC, "act_cast.cuh"), os.path.join(CSRC, "fp8_block.cuh"), os.path.join(CSRC, "fp8_index.h"), os.path.join(CSRC, "device_once.h"), os.path.join(CSRC, "kv_cache.cuh"), os.path.join(CSRC, "kv_index.h"), os.path.join(CSRC, "kv_attention.cuh"), os.path.join(HERE, "..", "include", "zqfp.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-fmad=true"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode:
            sys.stderr.write(out)
        failed |= pr.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.run([_nvcc(), "-shared", "-o", LIB, *objs, "-lcudart"], check=True)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
