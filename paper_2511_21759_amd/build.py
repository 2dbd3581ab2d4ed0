"""Builds libodb.so (HIP, gfx950 only) next to this file.

Every translation unit under csrc/ is compiled with hipcc for gfx950 and linked
into one shared library that exports the C ABI declared in include/odb.h.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libodb.so")
SOURCES = ["api.hip", "weights.hip", "rows.hip", "gemm.hip", "attn.hip", "paged.hip", "paged_attn.hip", "paged_quant.hip",
           "paged_attn_int8.hip", "paged_attn_e4m3.hip", "paged_api.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # MFMA results may stay in ordinary vector registers: without this the four-wave kernels (accumulators
         # beyond 256 registers) get their accumulators copied between the two register files around every MFMA
         "-mllvm", "-amdgpu-mfma-vgpr-form"]


def _hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: the library can only be built with ROCm installed")
    return exe


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), out))
    return out


def build_marshal() -> str:
    """_marshal: packs tensors into the C structures of calls where latency counts (csrc/marshal.cpp); host code against torch's headers."""
    import sysconfig
    import torch
    from torch.utils.cpp_extension import include_paths
    to = os.path.join(HERE, "_marshal.so")
    flags = ["-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    flags += ["-isystem" + p for p in include_paths() + [sysconfig.get_paths()["include"]]]
    libs = ["-L" + os.path.join(os.path.dirname(torch.__file__), "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python"]
    _run([shutil.which("g++") or "c++", *flags, os.path.join(CSRC, "marshal.cpp"), "-o", to + ".tmp", *libs])
    os.replace(to + ".tmp", to)
    return to


def build_library(verbose: bool = False, extra_flags=()) -> str:
    hipcc = _hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = [os.path.join(objdir, s.replace(".hip", ".o")) for s in SOURCES]

    def compile_one(i):
        return _run([hipcc, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, SOURCES[i]), "-o", objs[i]])

    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as ex:
        marshal = ex.submit(build_marshal)
        for out in ex.map(compile_one, range(len(SOURCES))):
            if verbose and out.strip():
                print(out, file=sys.stderr)
        marshal.result()
    tmp = LIB + ".tmp"
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
