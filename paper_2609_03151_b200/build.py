"""Build libbasp.so (sm_100a) in-tree with nvcc, and the binding's _marshal.so with g++.  `python -m paper_2609_03151_b200.build`."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libbasp.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
SOURCES = ["plan.cpp", "status.cu", "reshard.cu", "attn_fwd.cu", "attn_bwd.cu", "proj_gemm.cu", "layer.cu", "layer_static.cu",
           "norm_rope.cu", "ckpt.cu", "lm_loss.cu"]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    return "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "marshal.cpp"] + [os.path.join(ROOT, "include", "basp.h"), __file__]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-cudart", "static",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", LIB]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    return LIB


def build_marshal(force: bool = False) -> str:
    """The Python module that looks at a call's tensors (csrc/marshal.cpp)."""
    src = os.path.join(CSRC, "marshal.cpp")
    if not force and os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= max(os.path.getmtime(src), os.path.getmtime(__file__)):
        return MARSHAL
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                           "-I", sysconfig.get_paths()["include"], "-I", os.path.join(root, "include"),
                           "-I", os.path.join(root, "include", "torch", "csrc", "api", "include"), "-o", MARSHAL, src,
                           "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
                           "-Wl,-rpath," + os.path.join(root, "lib")])
    return MARSHAL


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_marshal(force="--force" in sys.argv))
