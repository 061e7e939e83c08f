"""In-tree build of the CUDA library (sm_100a only) and of the small module that looks at torch tensors."""
from __future__ import annotations

import glob
import importlib.util
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libans_b200.so")
FORM = os.path.join(HERE, "_ans_form.so")
FORM_MADE_FOR = os.path.join(HERE, "_build", "_ans_form.made_for")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "--fmad=false", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-shared",
]


def sources():
    c = os.path.join(HERE, "csrc")
    return sorted(glob.glob(os.path.join(c, "*.cu")) + glob.glob(os.path.join(c, "*.cpp")))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/ into libans_b200.so next to this file and, where torch is installed, the module that the operators on
    torch tensors need (build_form); returns the library's path."""
    if importlib.util.find_spec("torch"):
        build_form(force)
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


def form_interface() -> str:
    """What _ans_form.so is compiled against: torch's C++ objects and Python's, which it reads in place."""
    import torch
    return f"torch {torch.__version__}, {sys.implementation.cache_tag}"


def form_is_current() -> bool:
    """Whether _ans_form.so is of the source as it is and of the torch and Python that run."""
    source = os.path.join(HERE, "csrc", "torch", "ans_form.cpp")
    if not os.path.exists(FORM) or not os.path.exists(FORM_MADE_FOR) or os.path.getmtime(FORM) < os.path.getmtime(source):
        return False
    with open(FORM_MADE_FOR) as f:
        return f.read() == form_interface()


def build_form(force: bool = False) -> str:
    """Compile csrc/torch/ans_form.cpp into _ans_form.so next to this file; returns its path."""
    if not force and form_is_current():
        return FORM
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f'-DANS_MADE_FOR="{form_interface()}"',
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for d in [*include_paths(), sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", d]
    cmd += ["-o", FORM, os.path.join(HERE, "csrc", "torch", "ans_form.cpp"), "-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10"]
    subprocess.check_call(cmd)
    os.makedirs(os.path.dirname(FORM_MADE_FOR), exist_ok=True)
    with open(FORM_MADE_FOR, "w") as f:
        f.write(form_interface())
    return FORM


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
