"""Builds libbitnet_b200.so (sm_100a only) next to this file with nvcc, and the compiled part of the Python binding
(_binding.so, g++, where the headers of Python and torch are there).  No JIT cache, no fallback.

Every csrc/*.cu is compiled to an object under build/ (in parallel; an object is reused while it is newer than
its source and every header), then the objects are linked into the shared library.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(os.path.dirname(PKG), "include")
LIB = os.path.join(PKG, "libbitnet_b200.so")
OBJ_DIR = os.path.join(PKG, "build")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


BINDING = os.path.join(PKG, "_binding.so")
BINDING_SRC = os.path.join(CSRC, "binding.cpp")


def binding_tools():
    """What the binding is compiled with, as (compiler, include directories, library directory, versions, C++ ABI), or a text that says what is
    missing: a user of the C ABI alone needs neither a C++ compiler of its own nor the headers of Python and torch."""
    cxx = os.environ.get("CXX", "g++")
    if shutil.which(cxx.split()[0]) is None:
        return f"no C++ compiler ({cxx})"
    python = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(python, "Python.h")):
        return f"no Python.h in {python}"
    try:
        import torch
    except ImportError as e:
        return f"no torch ({e})"
    root = os.path.dirname(torch.__file__)
    if not os.path.exists(os.path.join(root, "include", "torch", "csrc", "autograd", "python_variable.h")):
        return f"no headers of torch in {root}"
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    dirs = [INCLUDE, python, os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
            os.path.join(cuda, "include")]
    abi = int(torch.compiled_with_cxx11_abi())
    return cxx, dirs, os.path.join(root, "lib"), f"python {sysconfig.get_python_version()} torch {torch.__version__} {root} abi {abi}", abi


def build_binding(force: bool = False):
    """csrc/binding.cpp against this Python and this torch (whose libraries are in the process already); again when its source, the header
    or either of those has changed.  None, with a warning, where something that it takes is missing: the calls it serves then raise."""
    tools = binding_tools()
    if isinstance(tools, str):
        warnings.warn(f"the compiled part of the Python binding is not built: {tools}")
        return None
    cxx, dirs, lib, versions, abi = tools
    newest = max(os.path.getmtime(f) for f in [BINDING_SRC, *glob.glob(os.path.join(INCLUDE, "*.h"))])
    made_for = os.path.join(OBJ_DIR, "binding_versions.txt")
    if not force and os.path.exists(BINDING) and os.path.getmtime(BINDING) > newest and os.path.exists(made_for):
        with open(made_for) as f:
            if f.read() == versions:
                return BINDING
    subprocess.run([*cxx.split(), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={abi}",
                    *[f"-I{d}" for d in dirs], "-o", BINDING, BINDING_SRC,
                    f"-L{lib}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", f"-Wl,-rpath,{lib}"], check=True)
    os.makedirs(OBJ_DIR, exist_ok=True)
    with open(made_for, "w") as f:
        f.write(versions)
    return BINDING


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def headers():
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in sources() + headers())


def build(force: bool = False, verbose: bool = False) -> str:
    """Both; the library whatever becomes of the binding."""
    with ThreadPoolExecutor(max_workers=1) as other:
        binding = other.submit(build_binding, force)
        build_library(force, verbose)
        binding.result()
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not (force or stale()):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    hdr_time = max(os.path.getmtime(h) for h in headers())
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src):
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        if (not force and not verbose and os.path.exists(obj)
                and os.path.getmtime(obj) > max(os.path.getmtime(src), hdr_time)):
            return obj
        subprocess.run([nvcc, *NVCC_FLAGS, *extra, "-I", INCLUDE, "-I", CSRC, "-c", "-o", obj, src], check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, sources()))
    subprocess.run([nvcc, "-shared", *NVCC_FLAGS[:2], "-o", LIB, *objs], check=True)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
