"""Build libmoesched.so (CUDA kernels + C ABI) for sm_100a with nvcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["api.cu", "mw_kernel.cu", "bvn_kernel.cu", "bvn_small.cu", "bvn_real_kernel.cu", "eval_kernel.cu", "order_kernel.cu", "bvn_static.cu", "probe.cu", "a2a_kernel.cu", "sinkhorn_kernel.cu",
           "route_kernel.cu", "slots_kernel.cu", "few_kernel.cu", "expert_kernel.cu", "norm_kernel.cu", "choose_kernel.cu", "rows_kernel.cu"]
HEADERS = [os.path.join(CSRC, "common.cuh"), os.path.join(CSRC, "peel.cuh"), os.path.join(CSRC, "small.cuh"), os.path.join(CSRC, "expert.cuh"), os.path.join(CSRC, "token.cuh"), os.path.join(CSRC, "schedule_read.h"), os.path.join(HERE, "..", "include", "moesched.h")]
LIB = os.path.join(HERE, "libmoesched.so")
LIB_CHECKED = os.path.join(HERE, "libmoesched_checked.so")   # the same sources with -DMOESCHED_CHECKED
BINDING = os.path.join(HERE, "_binding.so")                  # the compiled part of the Python binding (csrc/binding.cpp)


def _stale(lib) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def made_for() -> str:
    """What the compiled part of the binding goes with: it reads torch's C++ classes and Python's, of one version each."""
    import sysconfig

    import torch
    return f"moesched binding for torch {torch.__version__} {torch.version.git_version}, Python {sysconfig.get_config_var('SOABI')};"


def holds(path, text) -> bool:
    """Whether a compiled file has that text in it."""
    with open(path, "rb") as f:
        return text.encode() in f.read()


def build_binding(force: bool = False) -> str:
    """Compile the Python extension that calls the library (g++, against the installed torch; no GPU code). The file says what it was made for and how: one that was made
    for another torch or Python, or with other flags, is not up to date."""
    import sysconfig

    import torch
    source = os.path.join(CSRC, "binding.cpp")
    root = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    includes = [sysconfig.get_paths()["include"], os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                os.path.join(cuda, "include")]
    libs = os.path.join(root, "lib")
    flags = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
             *(f"-I{p}" for p in includes)]
    link = [f"-L{libs}", f"-Wl,-rpath,{libs}", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"]
    stamp = " ".join([made_for(), *flags, *link]).replace("\\", "/").replace('"', "'")
    newest = max(os.path.getmtime(p) for p in (source, os.path.join(HERE, "..", "include", "moesched.h")))
    if force or not os.path.exists(BINDING) or os.path.getmtime(BINDING) < newest or not holds(BINDING, stamp + "\0"):
        subprocess.run([*flags, f'-DMOESCHED_STAMP="{stamp}"', source, "-o", BINDING, *link], check=True)
    return BINDING


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile every source to an object file (in parallel, one nvcc per file) and link the library.
    checked=True builds the variant whose kernels range-check their data-dependent indices."""
    lib = LIB_CHECKED if checked else LIB
    if force or _stale(lib):
        _build_library(lib, verbose, checked)
    build_binding(force)             # (after the library, which does without it)
    return lib


def _build_library(lib, verbose, checked):
    from concurrent.futures import ThreadPoolExecutor
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objdir = os.path.join(HERE, "_build_checked" if checked else "_build")
    os.makedirs(objdir, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
    if checked:
        flags += ["-DMOESCHED_CHECKED"]
    if verbose:
        flags += ["-Xptxas", "-v"]

    def compile_one(src):
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        subprocess.run([nvcc, *flags, "-c", os.path.join(CSRC, src), "-o", obj], check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        objects = list(pool.map(compile_one, SOURCES))
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static", "-o", lib,
                    *objects], check=True)


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
