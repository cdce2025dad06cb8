"""Compile the CUDA sources into paper_2209_13258_b200/libosdp.so for sm_100a (in-tree)."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libosdp.so")
# Approximate functions and flushed denormals are fine for the GEMMs' epilogues; the optimiser's states, the norms'
# statistics and the int8 scales are computed with IEEE division and square root.
FAST_MATH_SOURCES = ["osdp_api.cu", "osdp_plan.cu", "osdp_experts.cu"]
SOURCES = FAST_MATH_SOURCES + ["osdp_step.cu", "osdp_block_norm.cu", "osdp_i8.cu", "osdp_route.cu", "osdp_expert_few.cu", "osdp_call.cu"]
HEADERS = ["osdp_gemm.cuh", "osdp_aux.cuh", "osdp_vec.cuh", "osdp_internal.h", "osdp_i8.h", "osdp_experts.h",
           os.path.join("..", "..", "include", "osdp.h")]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    with tempfile.TemporaryDirectory(prefix="osdp_build_") as objs:
        def compile_one(src):
            obj = os.path.join(objs, src + ".o")
            fast = ["--use_fast_math"] if src in FAST_MATH_SOURCES else []
            return obj, subprocess.run([nvcc] + NVCC_FLAGS + fast + ["-c", os.path.join(CSRC, src), "-o", obj],
                                       capture_output=True, text=True)

        with ThreadPoolExecutor(len(SOURCES)) as pool:
            done = list(pool.map(compile_one, SOURCES))
        steps = [r for _, r in done]
        if all(r.returncode == 0 for r in steps):
            steps.append(subprocess.run([nvcc] + NVCC_FLAGS + ["-shared"] + [o for o, _ in done] + ["-o", tmp],
                                        capture_output=True, text=True))
    failed = [r for r in steps if r.returncode != 0]
    if verbose or failed:
        for r in steps:
            print(r.stdout)
            print(r.stderr)
    if failed:
        raise RuntimeError("nvcc failed (exit %d)" % failed[0].returncode)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
