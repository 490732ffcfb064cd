"""Build the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdbt_b200.so")
SOURCES = ["dbt_api.cu", "dbt_ops.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "--expt-relaxed-constexpr"]


def _newest_source_mtime() -> float:
    t = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for f in os.listdir(root):
            if f.endswith((".cu", ".cuh", ".h")):
                t = max(t, os.path.getmtime(os.path.join(root, f)))
    return t


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    extra = os.environ.get("DBT_NVCC_EXTRA", "").split()  # experiment knobs (-D...), empty in normal builds
    flags = [*NVCC_FLAGS, *extra, *(["-Xptxas", "-v"] if verbose else [])]
    compile_flags = [f for f in flags if f != "-shared"]
    objects = [f"{tmp}.{i}.o" for i in range(len(SOURCES))]
    try:
        jobs = [subprocess.Popen([nvcc, *compile_flags, "-c", "-o", o, os.path.join(CSRC, s)]) for s, o in zip(SOURCES, objects)]
        for job, s in [(job, s) for job, s in zip(jobs, SOURCES) if job.wait() != 0]:
            raise subprocess.CalledProcessError(job.returncode, f"nvcc {s}")
        subprocess.run([nvcc, *flags, "-o", tmp, *objects, "-lcuda"], check=True)
        os.replace(tmp, LIB)
    finally:
        for o in objects:
            if os.path.exists(o):
                os.remove(o)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
