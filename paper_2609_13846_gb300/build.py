"""Compile libdtp.so (the C-ABI library of ``include/dtp.h``) for sm_103a with nvcc.

Each ``csrc/*.cu`` translation unit is compiled in parallel into
``_build/*.o`` and linked into ``paper_2609_13846_gb300/libdtp.so`` in the
source tree; ``csrc/tensor_lists.cpp``, the binding's reader of lists of tensors, becomes the
CPython module ``_tensor_lists.so`` beside it.  Run as ``python -m paper_2609_13846_gb300.build``.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import platform
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdtp.so")
LISTS = os.path.join(PKG, "_tensor_lists.so")
LISTS_SOURCE = os.path.join(CSRC, "tensor_lists.cpp")
LISTS_FOR = os.path.join(BUILD, "tensor_lists.for")     # the versions that the module was compiled against
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
              "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found")
    return exe


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _headers():
    return sorted(glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h")))


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
    cmd = [nvcc(), *ARCH, *NVCC_FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    log = os.path.join(BUILD, os.path.basename(src)[:-3] + ".ptxas.txt")
    with open(log, "w") as f:
        f.write(r.stderr)
    if verbose:
        sys.stderr.write(r.stderr)
    return obj


def versions() -> str:
    """What the module of tensor lists depends on: torch's C++ classes, CPython's, and the machine."""
    import torch
    return f"torch {torch.__version__}, {sys.implementation.cache_tag}, {platform.machine()}"


def lists_versions() -> str | None:
    """The versions that the module was compiled against, None where that is not known."""
    try:
        with open(LISTS_FOR) as f:
            return f.read()
    except OSError:
        return None


def _build_lists() -> None:
    import torch
    root = os.path.dirname(torch.__file__)
    lib = os.path.join(root, "lib")
    cuda = os.path.dirname(os.path.dirname(nvcc()))
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    tmp = LISTS + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-I{p}" for p in include), LISTS_SOURCE, "-o", tmp, f"-L{lib}", f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu",
           "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for {LISTS_SOURCE}:\n{r.stdout}\n{r.stderr}")
    os.makedirs(BUILD, exist_ok=True)
    if os.path.exists(LISTS_FOR):
        os.remove(LISTS_FOR)               # a module whose versions are not known is not loaded
    os.replace(tmp, LISTS)
    with open(LISTS_FOR + ".tmp", "w") as f:
        f.write(versions())
    os.replace(LISTS_FOR + ".tmp", LISTS_FOR)


def _stale(target: str, sources) -> bool:
    return not os.path.exists(target) or os.path.getmtime(target) < max(os.path.getmtime(p) for p in sources)


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libdtp.so and _tensor_lists.so where a source or header is newer, the latter also where torch or Python is another than
    it was compiled against; return the library's path."""
    srcs = _sources()
    lists = force or _stale(LISTS, [LISTS_SOURCE, __file__]) or lists_versions() != versions()
    library = force or _stale(LIB, srcs + _headers() + [__file__])
    with cf.ThreadPoolExecutor(max_workers=1) as beside:
        done = beside.submit(_build_lists) if lists else None
        if library:
            _build_library(srcs, verbose)
        if done:
            done.result()
    return LIB


def _build_library(srcs, verbose: bool) -> None:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    tmp = LIB + ".tmp"
    cmd = [nvcc(), *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
