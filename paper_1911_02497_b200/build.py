"""Builds the C-ABI shared library ``libcondensa_cstep.so`` next to this file
with nvcc for sm_100a. Run ``python -m paper_1911_02497_b200.build``."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcondensa_cstep.so")
OBJ = os.path.join(HERE, "build")
API_H = os.path.join("..", "..", "include", "condensa_cstep.h")
# each source with the headers it includes (they are compiled side by side)
SOURCES = {
    "api.cu": ["common.cuh", "ctx.cuh", "op_workspace.h", "ranges.h", "elementwise.cuh", "select.cuh", "structured.cuh", "fused.cuh", "fused_fast.cuh",
               "fused_blockg.cuh", "sample.cuh", "lstep.cuh", "thin.cuh", "small_select.cuh", "small_prune.cuh", API_H],
    "adapter.cu": ["common.cuh", "ctx.cuh", "op_workspace.h", "ranges.h", "adapter.cuh", "adapter_launch.cuh", API_H],
    "adapter_bf16.cu": ["common.cuh", "ctx.cuh", "op_workspace.h", "ranges.h", "adapter.cuh", "adapter_launch.cuh", "adapter_kernels.cuh", API_H],
    "adapter_f16.cu": ["common.cuh", "ctx.cuh", "op_workspace.h", "ranges.h", "adapter.cuh", "adapter_launch.cuh", "adapter_kernels.cuh", API_H],
    "adapter_f32.cu": ["common.cuh", "ctx.cuh", "op_workspace.h", "ranges.h", "adapter.cuh", "adapter_launch.cuh", "adapter_kernels.cuh", API_H],
    "adamw.cu": ["common.cuh", "ctx.cuh", "op_workspace.h", "ranges.h", "adamw.cuh", API_H],
}

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
              "--ftz=false", "--prec-div=true", "--prec-sqrt=true"]


def _deps(src):
    return [os.path.join(CSRC, f) for f in [src] + SOURCES[src]] + [os.path.abspath(__file__)]


def _older(path, deps) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def stale() -> bool:
    return any(_older(LIB, _deps(s)) for s in SOURCES)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    jobs, objects = [], []
    for src in SOURCES:
        obj = os.path.join(OBJ, src + ".o")
        objects.append(obj)
        if force or _older(obj, _deps(src)):
            cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj + ".tmp", os.path.join(CSRC, src)]
            jobs.append((src, obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for src, obj, p in jobs:
        out = p.communicate()[0]
        if verbose or p.returncode:
            sys.stderr.write(out)
        if p.returncode:
            failed.append(src)
        else:
            os.replace(obj + ".tmp", obj)
    if failed:
        raise RuntimeError("nvcc failed on %s" % ", ".join(failed))
    r = subprocess.run([nvcc] + NVCC_FLAGS + ["--shared", "-o", LIB + ".tmp"] + objects, capture_output=True, text=True)
    if r.returncode:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("nvcc failed linking %s" % LIB)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
