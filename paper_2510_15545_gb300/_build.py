"""Builds libtt.so (the C-ABI library of include/tt.h) in-tree with nvcc for
sm_103a. Translation units compile in parallel; the library links the shared
CUDA runtime, so a process that also runs PyTorch holds one runtime instance
(streams and events pass between the two unchanged)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from typing import List

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libtt.so")
SOURCES = ["api.cu", "align.cu", "rowpass.cu", "decide.cu", "noalloc.cu", "encode.cu", "shard.cu",
           "filter.cu", "nucleus.cu", "nucrow.cu", "pen.cu", "ops.cu", "logprob.cu",
           "distill.cu", "tree.cu", "rope.cu", "append.cu",
           "tree8.cu", "tree8_few.cu"]
HEADERS = ["tt_device.cuh", "tt_launch.h", "tt_shard.h", "tt_f2.cuh",
           "tt_ring.cuh", "tt_ops.h", "tt_umma.cuh", "tt_x2.cuh",
           "tt_rope.cuh", "tt_e4m3.cuh", "tt_tree8.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", shutil.which("nvcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libtt.so")


def _inputs() -> List[str]:
    files = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    files.append(os.path.join(ROOT, "include", "tt.h"))
    files.append(os.path.abspath(__file__))
    return files


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in _inputs())


def build(force: bool = False, verbose: bool = False, extra_flags: List[str] = ()) -> str:
    """Compiles every CUDA translation unit and links libtt.so; returns its path."""
    if not force and not is_stale():
        return LIB
    os.makedirs(OUT_DIR, exist_ok=True)
    cc = nvcc()
    common = ["-std=c++17", "-O3", "-lineinfo", *ARCH, "-Xcompiler", "-fPIC",
              "-I", os.path.join(ROOT, "include"), *extra_flags]
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(OUT_DIR, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = [cc, *common, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write(out.decode(errors="replace"))
        if p.returncode != 0:
            failed.append(src)
    if failed:
        raise RuntimeError("nvcc failed for: " + ", ".join(failed))
    tmp = LIB + ".tmp%d" % os.getpid()
    libdir = os.path.join(os.path.dirname(os.path.dirname(cc)), "lib64")
    subprocess.check_call([cc, "-shared", *ARCH, "-cudart", "shared", "-Xlinker", "-rpath",
                           "-Xlinker", libdir, "-o", tmp, *objs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv)
    print(LIB)
