"""Compile the HIP sources of the library for gfx950 into libnsa_sel.so next to this file."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = ["api.hip", "index.hip", "fwd.hip", "short.hip", "bwd.hip", "select.hip", "qouter.hip", "profile.hip",
           "cache_api.hip", "cache_append.hip", "cache_attend.hip", "cache_chunk.hip", "cache_read.hip", "rotary.hip"]
LIB = os.path.join(HERE, "libnsa_sel.so")
# -packed-fp32-ops: keep the compiler from forming packed fp32 instructions
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wall"]


# The same sources with cycle stamps in the pipelined 128-key backward kernel (see pipe_timing.py): a measuring build,
# loaded by that module only.
LIB_TIMING = os.path.join(HERE, "libnsa_sel_timing.so")


# The Python calls over a paged cache down to the library's C ABI (see csrc/bind_cache.cpp): a module of CPython and torch, beside the library.
LIB_NATIVE = os.path.join(HERE, "_cache_native.so")


def build_native(verbose: bool = False) -> str:
    """Needs the library (build()) to be there."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-isystem{p}" for p in (*include_paths(), sysconfig.get_paths()["include"])), os.path.join(HERE, "csrc", "bind_cache.cpp"),
           "-o", LIB_NATIVE, f"-L{torch_lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", f"-L{HERE}", "-l:libnsa_sel.so", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed")
    return LIB_NATIVE


def build(verbose: bool = False, timing: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    out = LIB_TIMING if timing else LIB
    cmd = [hipcc, *FLAGS, *(["-DNSA_PIPE_TIMING"] if timing else []), "-o", out,
           *[os.path.join(HERE, "csrc", s) for s in SOURCES]]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("hipcc failed")
    return out


if __name__ == "__main__":
    print(build(verbose=True))
    print(build(verbose=True, timing=True))
    print(build_native(verbose=True))
