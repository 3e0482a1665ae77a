"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the
operators' Python binding, a C++ extension on torch's headers, beside it."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
_SOURCE_NAMES = ("adascale.cu", "ops_embed.cu", "ops_distill.cu", "ops_norm.cu", "ops_position.cu", "ops_expert.cu",
                 "ops_clip.cu")
SOURCES = [os.path.join(_HERE, "csrc", name) for name in _SOURCE_NAMES]
HEADERS = [os.path.join(os.path.dirname(_HERE), "include", name) for name in ("adascale.h", "adascale_ops.h")] + \
          [os.path.join(_HERE, "csrc", name) for name in ("adascale_kernels.cuh", "ops_common.cuh")]
LIB = os.path.join(_HERE, "libadascale_b200.so")
OPS_SOURCE = os.path.join(_HERE, "csrc", "ops_binding.cpp")
OPS_LIB = os.path.join(_HERE, "_ops_binding.so")

NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared", "--threads", "0"]


def _nvcc():
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > built for p in SOURCES + HEADERS)


def ops_stale() -> bool:
    if not os.path.exists(OPS_LIB):
        return True
    built = os.path.getmtime(OPS_LIB)
    return any(os.path.getmtime(p) > built for p in (OPS_SOURCE, HEADERS[0], HEADERS[1]))


def _ops_command(out):
    """The binding links against the CUDA library beside it and against the torch that runs this."""
    import torch
    from torch.utils import cpp_extension
    flags = ["-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
             "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)]
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.sep in _nvcc() else "/usr/local/cuda"
    include = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    link = ["-L" + p for p in cpp_extension.library_paths()] + ["-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_cuda",
                                                               "-ltorch_python", "-L" + _HERE, "-l:" + os.path.basename(LIB),
                                                               "-Wl,-rpath,$ORIGIN"]
    return [os.environ.get("CXX", "g++")] + flags + ["-isystem" + p for p in include] + ["-o", out, OPS_SOURCE] + link


def build(force: bool = False, verbose: bool = False) -> str:
    if force or stale():
        tmp = LIB + ".%d.tmp" % os.getpid()
        cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES
        subprocess.check_call(cmd)
        os.replace(tmp, LIB)
    if force or ops_stale():
        tmp = OPS_LIB + ".%d.tmp" % os.getpid()
        subprocess.check_call(_ops_command(tmp))
        os.replace(tmp, OPS_LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
