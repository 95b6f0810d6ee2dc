"""Builds libfaasmoe.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the C extension in front of it."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "lib", "libfaasmoe.so")
CALLS = os.path.join(HERE, "lib", "_calls.so")          # marshalling of the context-free calls (CPython API only)
SOURCES = ["api.cu", "route.cu", "route_tc.cu", "dispatch.cu", "plan.cu", "experts_fma.cu", "experts_tc.cu", "combine.cu",
           "gate.cu", "addnorm.cu", "project.cu", "blocknorm.cu", "project_i8.cu", "balance.cu", "operators.cu"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "faasmoe.h")]
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and all(os.path.exists(f) and os.path.getmtime(f) >= _newest_source_mtime() for f in (LIB, CALLS)):
        return LIB
    os.makedirs(os.path.dirname(LIB), exist_ok=True)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "--threads", "0",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose:
        sys.stderr.write(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    cmd = ["gcc", "-O2", "-std=c11", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
           "-o", CALLS, os.path.join(CSRC, "calls.c")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("gcc failed:\n" + res.stdout + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
