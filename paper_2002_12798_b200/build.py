"""Builds libamap.so (host algebra + sm_100a kernels) in-tree with nvcc, and _serve_torch.so, the Python entry of the
serving operators, with g++ against PyTorch's headers."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libamap.so")
TORCH_ENTRY = os.path.join(HERE, "_serve_torch.so")
SOURCES = ["builder.cpp", "compose.cpp", "simplify.cpp", "plan_execute.cu", "consume.cu",
           "serve_common.cu", "serve_pages.cu", "serve_rope.cu", "serve_attend.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "serve_torch.cpp"] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [
        _nvcc(), "--threads", "0", "-std=c++17", "-O3", "-lineinfo", "-shared", "-Xcompiler", "-fPIC,-Wall,-Wextra",
        "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static",
        "-I", INCLUDE, "-I", CSRC, "-o", tmp,
    ] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


def _entry_stale(mark: str) -> bool:
    """Older than its sources, or of another PyTorch or Python (it carries the mark of those it was built against)."""
    if not os.path.exists(TORCH_ENTRY):
        return True
    deps = [os.path.join(CSRC, "serve_torch.cpp"), os.path.join(INCLUDE, "amap.h"), os.path.join(INCLUDE, "amap_serve.h")]
    if any(os.path.getmtime(d) > os.path.getmtime(TORCH_ENTRY) for d in deps):
        return True
    with open(TORCH_ENTRY, "rb") as f:
        return mark.encode() not in f.read()


def build_torch_entry(force: bool = False) -> str:
    """_serve_torch.so; libamap.so, which it calls, is built first and found beside it."""
    import sysconfig

    import torch

    lib = build_library()
    src = os.path.join(CSRC, "serve_torch.cpp")
    mark = "built against PyTorch %s, Python %s;" % (torch.__version__, sysconfig.get_config_var("SOABI"))
    if not force and not _entry_stale(mark):
        return TORCH_ENTRY
    there = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    tmp = TORCH_ENTRY + ".tmp%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-shared", "-fPIC", "-fvisibility=hidden", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi()]
    for d in [os.path.join(there, "include"), os.path.join(there, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], os.path.join(cuda, "include")]:
        cmd += ["-isystem", d]
    cmd += ["-I", INCLUDE, '-DSERVE_BUILT_AGAINST="%s"' % mark, src, "-o", tmp]
    cmd += ["-L", os.path.join(there, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-L", HERE, "-l:" + os.path.basename(lib), "-Wl,-rpath,$ORIGIN"]
    subprocess.check_call(cmd)
    os.replace(tmp, TORCH_ENTRY)
    return TORCH_ENTRY


if __name__ == "__main__":
    build_torch_entry(force="--force" in sys.argv)
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
