"""Build libpatchkv.so in-tree with nvcc for sm_100a (no torch headers involved)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpatchkv.so")
SOURCES = ["context.cu", "restore.cu", "select.cu", "host_restore.cu", "writer.cu", "cache.cu", "rotary.cu", "evict.cu", "attention.cu", "mass.cu",
           "attention_split_64.cu", "attention_split_128.cu", "attention_rows_64.cu", "attention_rows_128.cu",
           "mass_split_64.cu", "mass_split_128.cu", "mass_rows_64.cu", "mass_rows_128.cu"]
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler",
         "-fPIC,-fvisibility=hidden", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _newest_source_mtime() -> float:
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "patchkv.h")]
    return max(os.path.getmtime(f) for f in files)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".{os.getpid()}.tmp"
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(os.cpu_count() or 1) as pool:
        # One nvcc per source, all at once.  (--split-compile is as quick, but cuts a module anew each time: the same attention
        # sources then gave objects of 10 to 13 MB, and one decode call took 15.5 us with some and 17.4 us with others.)
        def compile_one(source: str) -> str:
            obj = os.path.join(objects, source + ".o")
            subprocess.check_call([nvcc, *(["-Xptxas", "-v"] if verbose else []), *FLAGS, "-c", "-o", obj, os.path.join(CSRC, source)])
            return obj
        objs = list(pool.map(compile_one, SOURCES))
        subprocess.check_call([nvcc, *FLAGS, "-shared", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
