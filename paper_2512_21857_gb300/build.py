"""Builds libadt.so (CUDA for sm_103a) in-tree, next to this file, and
_marshal.so, the binding's C++ part (for the torch that is installed).

Every translation unit is compiled in parallel with nvcc, then linked into a
shared library with the CUDA runtime linked statically.  Run
``python -m paper_2512_21857_gb300.build`` or call ``build()``.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB_PATH = os.path.join(PKG, "libadt.so")
MARSHAL_PATH = os.path.join(PKG, "_marshal.so")

ARCH_FLAGS = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-O3", "-I", INCLUDE, "-I", CSRC]


def nvcc() -> str:
    cand = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libadt")
    return cand


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cpp")))


def _compile(src: str, extra) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    deps = [src] + [os.path.join(CSRC, h) for h in os.listdir(CSRC) if h.endswith((".cuh", ".h"))]
    deps.append(os.path.join(INCLUDE, "adt.h"))
    if os.path.exists(obj) and all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in deps):
        return obj
    cmd = [nvcc()] + ARCH_FLAGS + COMMON_FLAGS + list(extra) + ["-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed for {os.path.basename(src)}:\n{res.stdout}\n{res.stderr}")
    if res.stderr.strip() and os.environ.get("ADT_BUILD_VERBOSE"):
        sys.stderr.write(res.stderr)
    return obj


def _marshal() -> str:
    """The binding's C++ part: against torch's headers, with the host compiler."""
    src = os.path.join(CSRC, "marshal.cc")
    import torch
    home = os.path.dirname(os.path.abspath(torch.__file__))
    stamp = os.path.join(BUILD_DIR, "marshal.torch")  # rebuilt for another torch
    deps = [src, os.path.join(INCLUDE, "adt.h")]
    if os.path.exists(MARSHAL_PATH) and all(os.path.getmtime(MARSHAL_PATH) >= os.path.getmtime(d) for d in deps) and \
            os.path.exists(stamp) and open(stamp).read() == torch.__version__:
        return MARSHAL_PATH
    tmp = MARSHAL_PATH + ".tmp"
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    cmd = [os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
           "-I", sysconfig.get_paths()["include"], "-I", os.path.join(home, "include"),
           "-I", os.path.join(home, "include", "torch", "csrc", "api", "include"), "-I", cuda, src, "-o", tmp,
           "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ldl"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"the compiler failed for {os.path.basename(src)}:\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, MARSHAL_PATH)
    with open(stamp, "w") as f:
        f.write(torch.__version__)
    return MARSHAL_PATH


def build(verbose: bool = False, extra_flags=()) -> str:
    """Compiles the library if any source is newer than it; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = sources()
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as ex:
        marshal = ex.submit(_marshal)
        objs = list(ex.map(lambda s: _compile(s, extra_flags), srcs))
        marshal.result()
    if not os.path.exists(LIB_PATH) or any(os.path.getmtime(o) > os.path.getmtime(LIB_PATH) for o in objs):
        tmp = LIB_PATH + ".tmp"
        cmd = [nvcc()] + ARCH_FLAGS + ["-shared", "-o", tmp] + objs
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
        os.replace(tmp, LIB_PATH)
    if verbose:
        print(f"built {LIB_PATH}")
    return LIB_PATH


if __name__ == "__main__":
    build(verbose=True)
