"""In-tree build of the CUDA library (nvcc, sm_100a only)."""
from __future__ import annotations

import concurrent.futures
import hashlib
import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libnk_gemm.so")
SOURCES = ["nk_gemm.cu", "nk_grouped.cu", "grouped_rows.cu", "grouped_weights.cu", "grouped_lora.cu",
           "nk_route.cu", "nk_lora.cu", "nk_pack.cu", "nk_mx.cu",
           "mx_nv.cu", "mx_mx.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


STAMP = LIB + ".srchash"


def _reach(path: str, seen: set) -> set:
    """The file and everything it includes by a quoted name."""
    path = os.path.normpath(path)
    if path not in seen:
        seen.add(path)
        with open(path) as f:
            for name in re.findall(r'^\s*#include "([^"]+)"', f.read(), re.M):
                _reach(os.path.join(os.path.dirname(path), name), seen)
    return seen


def source_hash(sources=None) -> str:
    """Hash of everything the library (or these of its sources) is compiled from, and of the flags: a
    check-out or a copy of the tree may not keep file times, so staleness is decided on contents."""
    h = hashlib.sha256(" ".join(NVCC_FLAGS).encode())
    files = set()
    for s in sources or SOURCES:
        _reach(os.path.join(CSRC, s), files)
    for path in sorted(files):
        h.update(os.path.basename(path).encode())
        with open(path, "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def _stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(STAMP):
        return True
    with open(STAMP) as f:
        return f.read().strip() != source_hash()


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libnk_gemm.so next to this file (unless it is already built from
    the sources as they are now); returns its path.  Objects are kept by the hash of what they are
    compiled from, so a change rebuilds the files that it reaches; `force` compiles them all."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = list(NVCC_FLAGS)
    if verbose:
        flags += ["-Xptxas", "-v"]
    os.makedirs(OBJ, exist_ok=True)

    def compile_one(source):
        obj = os.path.join(OBJ, f"{source}.{source_hash([source])[:16]}.o")
        if force or verbose or not os.path.exists(obj):
            tmp = f"{obj}.{os.getpid()}.tmp.o"
            subprocess.check_call([nvcc] + flags + ["-c", "-o", tmp, os.path.join(CSRC, source)])
            os.replace(tmp, obj)
        return obj

    with concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = list(pool.map(compile_one, SOURCES))
    tmp = LIB + f".{os.getpid()}.tmp"
    subprocess.check_call([nvcc] + NVCC_FLAGS + ["-shared", "-o", tmp] + objects + ["-lcudart"])
    os.replace(tmp, LIB)
    with open(STAMP + f".{os.getpid()}.tmp", "w") as f:
        f.write(source_hash())
    os.replace(STAMP + f".{os.getpid()}.tmp", STAMP)
    for name in os.listdir(OBJ):
        if os.path.join(OBJ, name) not in objects and not name.endswith(".tmp.o"):
            try:
                os.remove(os.path.join(OBJ, name))
            except FileNotFoundError:
                pass
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
