"""Builds libmpq.so (the C-ABI library) in-tree from csrc/*.cu with nvcc for sm_103a.

Translation units compile in parallel, then link into one shared library with the CUDA runtime
linked statically.  The native marshalling of the serving calls (csrc/bind/) is a Python extension of its
own, _serve_binding.so, compiled (by the host compiler that nvcc uses too) against the torch that imports it,
and again when that torch or the Python changes.  Run ``python -m paper_2002_09049_gb300._build`` or call
``build()``.
``build(checked=True)`` (``--checked``) builds the checked library, libmpq_checked.so: the same
sources with -DMPQ_CHECK_BOUNDS, whose kernels count and skip out-of-range accesses.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig
import threading
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libmpq.so")
CHECKED_LIB = os.path.join(PKG, "libmpq_checked.so")
BINDING = os.path.join(PKG, "_serve_binding.so")
BINDING_FOR = os.path.join(BUILD, "serve_binding.for")   # what it was compiled against
ROOT = os.path.dirname(PKG)
INCLUDE = os.path.join(ROOT, "include")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-O2", "-I", INCLUDE,
              "-Xptxas", "-warn-spills"]
_lock = threading.Lock()


def nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libmpq.so")
    return cand


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + [os.path.join(INCLUDE, "mpq.h")]


def up_to_date(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return False
    t = os.path.getmtime(lib)
    return all(os.path.getmtime(p) <= t for p in _deps())


def _binding_against() -> str:
    """What the extension depends on besides its sources: this Python's and this torch's C++ interfaces."""
    import torch
    return "\n".join((sysconfig.get_config_var("SOABI") or sys.version, torch.__version__,
                      str(int(torch._C._GLIBCXX_USE_CXX11_ABI))))


def binding_fits() -> bool:
    """Whether the extension was compiled against this Python and this torch."""
    try:
        with open(BINDING_FOR) as f:
            return f.read() == _binding_against()
    except FileNotFoundError:
        return False


def _binding_up_to_date() -> bool:
    src = os.path.join(CSRC, "bind", "serve_binding.cpp")
    return os.path.exists(BINDING) and binding_fits() and all(
        os.path.getmtime(p) <= os.path.getmtime(BINDING)
        for p in (src, os.path.join(INCLUDE, "mpq.h")))


def _build_binding(exe: str) -> None:
    """Compile csrc/bind/serve_binding.cpp -> _serve_binding.so with the host compiler."""
    import torch
    home = os.path.dirname(torch.__file__)
    inc = [os.path.join(home, "include"),
           os.path.join(home, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(exe))), "include"),
           sysconfig.get_paths()["include"], INCLUDE]
    libs = os.path.join(home, "lib")
    tmp = BINDING + f".{os.getpid()}.tmp"
    cmd = [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[f"-I{p}" for p in inc], os.path.join(CSRC, "bind", "serve_binding.cpp"), "-o", tmp,
           f"-L{libs}", f"-Wl,-rpath,{libs}", "-ltorch_python", "-ltorch", "-ltorch_cpu",
           "-ltorch_cuda", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"compiling the serving calls' binding failed:\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, BINDING)
    os.makedirs(BUILD, exist_ok=True)
    tmp = BINDING_FOR + f".{os.getpid()}.tmp"
    with open(tmp, "w") as f:
        f.write(_binding_against())
    os.replace(tmp, BINDING_FOR)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False,
          checked: bool = False) -> str:
    """Compile csrc/*.cu -> libmpq.so, or with checked=True -> libmpq_checked.so (skipped when
    up to date).  Returns the library path."""
    lib = CHECKED_LIB if checked else LIB
    obj_dir = os.path.join(BUILD, "checked") if checked else BUILD
    with _lock:
        stale = force or not up_to_date(lib)
        bind = force or not _binding_up_to_date()
        if not (stale or bind):
            return lib
        exe = nvcc()
        if not stale:
            _build_binding(exe)
            return lib
        os.makedirs(obj_dir, exist_ok=True)
        extra = ["-Xptxas", "-v"] if ptxas_info else []
        if checked:
            extra += ["-DMPQ_CHECK_BOUNDS"]

        def compile_one(src):
            obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
            cmd = [exe, *ARCH, *NVCC_FLAGS, *extra, "-c", src, "-o", obj]
            res = subprocess.run(cmd, capture_output=True, text=True)
            if res.returncode != 0:
                raise RuntimeError(f"nvcc failed on {src}:\n{res.stdout}\n{res.stderr}")
            if verbose or ptxas_info:
                sys.stderr.write(res.stdout + res.stderr)
            return obj

        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 4)) as ex:
            extension = ex.submit(_build_binding, exe) if bind else None
            objs = list(ex.map(compile_one, _sources()))
            if extension:
                extension.result()
        tmp = lib + f".{os.getpid()}.tmp"
        cmd = [exe, *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
        os.replace(tmp, lib)
        return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, ptxas_info="--ptxas" in sys.argv,
                checked="--checked" in sys.argv))
