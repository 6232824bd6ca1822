"""Builds ``libmala.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU), and beside it ``_native.so``, the marshalling
of the calls that serving steps wait for, with g++ against torch."""
from __future__ import annotations

import contextlib
import os
import shutil
import subprocess
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", n) for n in ("mala_api.cu", "mala_bias.cu", "mala_cache.cu", "mala_rotary.cu", "mala_rotary_write8.cu",
                                                "mala_scaled.cu")]
LIB = os.path.join(HERE, "libmala.so")
NATIVE_SRC = os.path.join(HERE, "csrc", "mala_native.cpp")
NATIVE = os.path.join(HERE, "_native.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")


def _up_to_date(built: str, sources) -> bool:
    return os.path.exists(built) and os.path.getmtime(built) >= max(map(os.path.getmtime, sources))


def _sources():
    files = [os.path.join(root, f) for root in (os.path.join(HERE, "csrc"), INCLUDE) for f in os.listdir(root)]
    return [f for f in files if f != NATIVE_SRC]


def _native_for() -> str:
    """What _native.so is bound to beside its sources: a torch, whose C++ types it shares and whose libraries it names, and an interpreter."""
    import torch
    return "\n".join((torch.__version__, os.path.dirname(torch.__file__), sysconfig.get_config_var("SOABI") or "")) + "\n"


def _native_command(out: str):
    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    libs = os.path.join(home, "lib")
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] +
            [f"-I{p}" for p in include] + [NATIVE_SRC, "-o", out, f"-L{libs}", "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10",
                                           f"-Wl,-rpath,{libs}", f"-L{HERE}", "-l:libmala.so", "-Wl,-rpath,$ORIGIN"])


@contextlib.contextmanager
def _replacing(path: str):
    """A name beside `path` to write to; what stands there is `path` afterwards, unless writing fails (a part of a file would count as up to date)."""
    tmp = f"{path}.{os.getpid()}.tmp"
    try:
        yield tmp
        os.replace(tmp, path)
    finally:
        if os.path.exists(tmp):
            os.remove(tmp)


def _native_record() -> str:
    return NATIVE + ".for"


def _native_up_to_date() -> bool:
    if not _up_to_date(NATIVE, [NATIVE_SRC, os.path.join(INCLUDE, "mala.h")]) or not os.path.exists(_native_record()):
        return False
    with open(_native_record()) as f:
        return f.read() == _native_for()


def build(force: bool = False, verbose: bool = False) -> str:
    if force or not _up_to_date(LIB, _sources()):
        _build_library(verbose)
    if force or not _native_up_to_date():
        with _replacing(NATIVE) as out:
            subprocess.check_call(_native_command(out))
        with _replacing(_native_record()) as out, open(out, "w") as f:
            f.write(_native_for())
    return LIB


def _build_library(verbose: bool) -> None:
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
        with _replacing(LIB) as out:
            subprocess.check_call(nvcc[:3] + ["-shared", "-o", out] + objs + ["-ldl"])


if __name__ == "__main__":
    print(build(force=True, verbose=True))
