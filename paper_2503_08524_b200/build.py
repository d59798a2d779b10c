"""Builds libd3.so (the CUDA library behind the C ABI of include/d3.h) in-tree
with nvcc for sm_100a, and _paged_call.*.so and _block_call.*.so (the Python side of the
paged and of the 8-bit block operators' calls, csrc/*_call.cpp) with g++.  No GPU is needed to build."""
from __future__ import annotations

import glob
import os
import re
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libd3.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ (one nvcc per file, in parallel) and link libd3.so;
    returns the library path."""
    if not force and not _stale():
        return LIB
    from concurrent.futures import ThreadPoolExecutor
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
             "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    headers = glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        if (not force and not verbose and os.path.exists(obj)
                and os.path.getmtime(obj) > max(os.path.getmtime(src), newest_header)):
            return obj, ""
        res = subprocess.run([NVCC] + flags + ["-c", src, "-o", obj], capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed on " + src + ":\n" + res.stdout + res.stderr)
        return obj, res.stderr

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        done = list(pool.map(compile_one, sources()))
    if verbose:
        for _, err in done:
            sys.stderr.write(err)
    res = subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB] +
                         [obj for obj, _ in done], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stdout + res.stderr)
    return LIB


CALLS = ("paged_call", "block_call")      # extension modules, by their source


def call_path(name: str = "paged_call") -> str:
    """Where an extension module lies: it reads torch's objects, so its name says what it was built for."""
    import torch
    made_for = "-".join((sys.implementation.cache_tag, "torch" + torch.__version__, "cxx11abi%d" % torch._C._GLIBCXX_USE_CXX11_ABI))
    return os.path.join(PKG, "_" + name + "." + re.sub(r"[^0-9A-Za-z-]", "_", made_for) + ".so")


def build_call(force: bool = False, name: str = "paged_call") -> str:
    """Compile and link an extension module that makes operators' calls (default: the paged ones'); returns its path."""
    src, header = os.path.join(CSRC, name + ".cpp"), os.path.join(ROOT, "include", "d3.h")
    out = call_path(name)
    if not force and os.path.exists(out) and os.path.getmtime(out) > max(os.path.getmtime(src), os.path.getmtime(header)):
        return out
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(NVCC))
    # a file of this process's own until it is whole: ranks that import a fresh checkout build it side by side
    handle, made = tempfile.mkstemp(dir=os.path.dirname(out), prefix="_" + name + ".", suffix=".new")
    os.close(handle)
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(base, "include"),
           "-I", os.path.join(base, "include", "torch", "csrc", "api", "include"), "-I", os.path.join(cuda, "include"), src, "-o", made,
           "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    try:
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("g++ failed on " + src + ":\n" + res.stdout + res.stderr)
        os.chmod(made, 0o755)      # (mkstemp's files are the owner's alone)
        os.replace(made, out)
    finally:
        if os.path.exists(made):
            os.remove(made)
    return out


def load_call(name: str = "paged_call"):
    """An extension module, built if need be."""
    import importlib.util
    spec = importlib.util.spec_from_file_location(__package__ + "._" + name, build_call(name=name))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
    for call in CALLS:
        print(build_call(force=True, name=call))
