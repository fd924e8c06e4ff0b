"""Build libebd.so (the C ABI of include/ebd.h) for GB300, in-tree.

Each CUDA translation unit is compiled for sm_103a in parallel, then linked
into ``paper_2607_21475_gb300/_build/libebd.so``.  A content hash of the
sources and flags skips the build when nothing changed.  The marshalling of the serving
calls (csrc/binding.cpp) is a Python extension beside it, ``_build/ebd_call.so``,
compiled by g++ against the headers of the torch that is installed.
"""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(BUILD, "libebd.so")
CALL = os.path.join(BUILD, "ebd_call.so")
BINDING = os.path.join(CSRC, "binding.cpp")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--use_fast_math",
              "-Xptxas", "-O3", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    cand = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found; the CUDA 13 toolkit is required to build libebd")
    return cand


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _torch_root() -> str | None:
    from importlib.util import find_spec
    spec = find_spec("torch")
    return os.path.dirname(spec.origin) if spec is not None and spec.origin else None


def _compile_binding() -> None:
    """The extension of csrc/binding.cpp, for this interpreter and this torch."""
    if os.path.exists(CALL):
        os.remove(CALL)  # (one of other sources would marshal for a library that is gone)
    root, nvcc = _torch_root(), _nvcc()
    if root is None:
        raise RuntimeError("torch not found; the binding is compiled against its headers")
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
    tmp = CALL + ".tmp"
    include = [os.path.join(root, "include"),
               os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    lib = os.path.join(root, "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w",
           *[x for d in include for x in ("-isystem", d)], BINDING, "-o", tmp, "-L", lib,
           "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda",
           f"-Wl,-rpath,{lib}"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"the binding needs a C++ compiler: {e}") from e
    if r.returncode != 0:
        raise RuntimeError(f"the binding failed to compile:\n{r.stderr[-4000:]}")
    os.replace(tmp, CALL)


def _digest(extra_flags) -> str:
    h = hashlib.sha256()
    # the binding is for one interpreter and one torch
    root = _torch_root() or ""
    h.update((sys.version + root).encode())
    version = os.path.join(root, "version.py")
    files = [BINDING] + ([version] if root and os.path.exists(version) else [])
    files += _sources() + sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC)
                                 if f.endswith((".cuh", ".h")))
    files.append(os.path.join(INCLUDE, "ebd.h"))
    for f in files:
        h.update(f.encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(ARCH + NVCC_FLAGS + list(extra_flags)).encode())
    return h.hexdigest()


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile the CUDA sources and link libebd.so, and compile the binding; returns the
    library path.  Where the binding does not compile, the library is there all the same:
    the calls that go through ctypes, and C programs, do without it."""
    os.makedirs(BUILD, exist_ok=True)
    stamp = os.path.join(BUILD, "libebd.stamp")
    dig = _digest(extra_flags)
    if not force and os.path.exists(LIB) and os.path.exists(CALL) and os.path.exists(stamp):
        with open(stamp) as fh:
            if fh.read().strip() == dig:
                return LIB
    nvcc = _nvcc()
    srcs = _sources()
    objs = [os.path.join(BUILD, os.path.basename(s)[:-3] + ".o") for s in srcs]

    def compile_one(src_obj):
        src, obj = src_obj
        cmd = [nvcc, *ARCH, *NVCC_FLAGS, *extra_flags, "-I", INCLUDE, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {os.path.basename(src)}:\n{r.stderr}")
        if verbose and r.stderr:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(srcs) + 1, os.cpu_count() or 4)) as ex:
        binding = ex.submit(_compile_binding)
        list(ex.map(compile_one, zip(srcs, objs)))
    tmp = LIB + ".tmp"
    cmd = [nvcc, *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link of libebd.so failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if binding.exception() is not None:
        raise RuntimeError(f"{LIB} is built, the binding of the serving calls is not") \
            from binding.exception()
    with open(stamp, "w") as fh:
        fh.write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
