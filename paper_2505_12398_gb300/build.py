"""Build the in-tree CUDA library ``libtv.so`` for sm_103a (GB300).

Usage: ``python -m paper_2505_12398_gb300.build`` (or ``build()`` from
Python).  Each translation unit is compiled in parallel with nvcc, then
linked into a shared library next to this file.  Rebuilds only when a source
is newer than the library.  Concurrent callers (e.g. the ranks of a multi-GPU
run) are serialised by a file lock, and a caller that waited finds the library
built.
"""

import fcntl
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libtv.so")
SOURCES = ["tv_api.cu", "tv_kernels.cu", "tv_tree.cu", "tv_flow.cu", "tv_noalloc.cu", "tv_gemm.cu",
           "tv_bonus.cu",
           "tv_draft.cu", "tv_gemm8.cu", "tv_norm.cu", "tv_logits.cu"]
HEADERS = ["tv_device.cuh", "tv_launch.h", "tv_ptx.cuh", "tv_control.cuh", "tv_umma.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall"]


def _nvcc():
    nvcc = shutil.which("nvcc")
    if nvcc:
        return nvcc
    cand = "/usr/local/cuda/bin/nvcc"
    if os.path.exists(cand):
        return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libtv.so")


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    deps.append(os.path.join(ROOT, "include", "tv.h"))
    deps.append(os.path.abspath(__file__))
    return any(os.path.getmtime(d) > t for d in deps)


def with_build_lock(fn):
    """Runs fn() holding the build folder's exclusive lock (across processes)."""
    os.makedirs(BUILD, exist_ok=True)
    with open(os.path.join(BUILD, ".lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        try:
            return fn()
        finally:
            fcntl.flock(lock, fcntl.LOCK_UN)


def build(force=False, verbose=False):
    """Compile libtv.so if needed; returns its path."""
    if not force and not _stale():
        return LIB
    return with_build_lock(lambda: LIB if (not force and not _stale())
                           else _build(verbose))


def _build(verbose):
    nvcc = _nvcc()
    os.makedirs(BUILD, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        cmd = [nvcc, *ARCH, *FLAGS, "-I", os.path.join(ROOT, "include"), "-c",
               os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-lcudart", "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
