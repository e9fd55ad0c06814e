"""Builds libb200gemm.so in-tree with nvcc for sm_100a (cross-compiles without a GPU).

    python -m paper_2608_10103_b200.build [--force] [--verbose]

One object per .cu file, compiled side by side, linked into one shared library; and the
argument marshalling of the Python binding (csrc/marshal.cpp) as an extension module beside it.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libb200gemm.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
INCLUDE = os.path.join(os.path.dirname(PKG), "include")

NVCC_FLAGS = [
    "-std=c++17", "-O3", "-lineinfo",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-Xcompiler", "-fPIC",
]
LINK_FLAGS = ["-shared", "-cudart", "shared"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _marshal_command(out: str):
    """Host code only: torch's headers, no CUDA compiler."""
    import torch
    root = os.path.dirname(torch.__file__)
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], "/usr/local/cuda/include"]
    libs = os.path.join(root, "lib")
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    return (["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-fvisibility=hidden",
             "-D_GLIBCXX_USE_CXX11_ABI=%d" % abi] + [x for d in include for x in ("-isystem", d)] +
            ["-o", out, os.path.join(CSRC, "marshal.cpp"), "-L" + libs, "-Wl,-rpath," + libs,
             "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])


def _stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(MARSHAL):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(MARSHAL))
    deps = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = ["-Xptxas", "-v"] if verbose else []
    with tempfile.TemporaryDirectory(prefix="b200gemm_build_") as tmp:
        objects, running = [], []
        for src in sources():
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            cmd = [nvcc] + NVCC_FLAGS + extra + ["-c", "-o", obj, src]
            running.append((cmd, subprocess.Popen(cmd)))
            objects.append(obj)
        marshal = MARSHAL + ".tmp.%d" % os.getpid()
        cmd = _marshal_command(marshal)
        running.append((cmd, subprocess.Popen(cmd)))
        codes = [(cmd, p.wait()) for cmd, p in running]
        for cmd, rc in codes:
            if rc != 0:
                raise subprocess.CalledProcessError(rc, cmd)
        out = LIB + ".tmp.%d" % os.getpid()
        subprocess.check_call([nvcc] + NVCC_FLAGS + LINK_FLAGS + ["-o", out] + objects)
    os.replace(out, LIB)
    os.replace(marshal, MARSHAL)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
