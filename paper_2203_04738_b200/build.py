"""Builds the CUDA library in-tree for sm_100a:  python -m paper_2203_04738_b200.build"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmgrit_gru.so")
SOURCES = ["api.cu", "simt_kernels.cu", "f32_solve.cu", "stream_kernels.cu", "umma_engine.cu", "serial_kernels.cu", "scan_kernels.cu",
           *(f"scan_{t}_{m}.cu" for t in ("f32", "bf16", "f16") for m in ("cells", "open", "given")), "logit_kernels.cu"]
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "mgrit_gru.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = os.environ.get("MGRIT_GRU_NVCC_FLAGS", "").split()      # e.g. -D switches of kernel variants under study
    with tempfile.TemporaryDirectory() as tmp:                      # every source by itself, all at once, then one link
        objs = [os.path.join(tmp, s + ".o") for s in SOURCES]
        cmds = [[nvcc] + FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", o, os.path.join(CSRC, s)] for s, o in zip(SOURCES, objs)]
        with ThreadPoolExecutor(min(len(cmds), os.cpu_count() or 1)) as pool:
            runs = list(pool.map(lambda c: subprocess.run(c, capture_output=True, text=True), cmds))
        if all(r.returncode == 0 for r in runs):
            runs.append(subprocess.run([nvcc] + FLAGS + extra + ["-shared", "-o", LIB] + objs, capture_output=True, text=True))
    failed = any(r.returncode != 0 for r in runs)
    if verbose or failed:
        sys.stderr.write("".join(r.stdout + r.stderr for r in runs))
    if failed:
        raise RuntimeError("nvcc failed building libmgrit_gru.so")
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
