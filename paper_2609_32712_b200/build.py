"""Builds ``libmala.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", n) for n in ("mala_api.cu", "mala_bias.cu", "mala_cache.cu")]
LIB = os.path.join(HERE, "libmala.so")


def _newest_source_mtime() -> float:
    t = 0.0
    for root in (os.path.join(HERE, "csrc"), os.path.join(os.path.dirname(HERE), "include")):
        for f in os.listdir(root):
            t = max(t, os.path.getmtime(os.path.join(root, f)))
    return t


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    # (one nvcc per source, side by side; the objects go to a folder that does not outlive the call)
    nvcc = ["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC"]
    if verbose:
        nvcc.append("-Xptxas=-v")
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SRCS]
        jobs = [subprocess.Popen(nvcc + ["-c", "-o", o, s]) for o, s in zip(objs, SRCS)]
        codes = [j.wait() for j in jobs]
        if any(codes):
            raise RuntimeError(f"nvcc failed: {[os.path.basename(s) for s, c in zip(SRCS, codes) if c]}")
        subprocess.check_call(nvcc[:3] + ["-shared", "-o", LIB] + objs + ["-ldl"])
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
