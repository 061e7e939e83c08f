"""In-tree build of the CUDA library (sm_100a only) and of the small module that looks at torch tensors."""
from __future__ import annotations

import glob
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libans_b200.so")
FORM = os.path.join(HERE, "_ans_form.so")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "--fmad=false", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-shared",
]


def sources():
    c = os.path.join(HERE, "csrc")
    return sorted(glob.glob(os.path.join(c, "*.cu")) + glob.glob(os.path.join(c, "*.cpp")))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/ into libans_b200.so next to this file; returns its path."""
    deps = sources() + glob.glob(os.path.join(HERE, "csrc", "*.cuh")) + \
        glob.glob(os.path.join(ROOT, "include", "*.h"))
    if not force and os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in deps):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += ["-o", LIB, *sources()]
    subprocess.check_call(cmd)
    return LIB


def build_form(force: bool = False) -> str:
    """Compile csrc/torch/ans_form.cpp into _ans_form.so next to this file; returns its path."""
    import sysconfig
    source = os.path.join(HERE, "csrc", "torch", "ans_form.cpp")
    if not force and os.path.exists(FORM) and os.path.getmtime(FORM) >= os.path.getmtime(source):
        return FORM
    import torch
    from torch.utils.cpp_extension import include_paths
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for d in [*include_paths(), sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", d]
    cmd += ["-o", FORM, source, "-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10"]
    subprocess.check_call(cmd)
    return FORM


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
    print(build_form(force=True))
