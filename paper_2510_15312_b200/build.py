"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsdv.so")
_UNITS = ["sdv.cu", "paged.cu"]   # compiled side by side
_SOURCES = _UNITS + ["forward.cuh", "dense.cuh", "device_once.h", "layout.cuh", "paged.cuh", "ptx.cuh", "small_gemm.cuh", "small_kernels.cuh",
                     "tensor_map.h", "tree_attention.cuh", "tree_plan.h", "verify_sampled.cuh"]


HASH_PATH = LIB_PATH + ".srchash"


def _source_hash() -> str:
    """Digest of every source the library is built from (file times do not survive a checkout or a copy)."""
    import hashlib
    h = hashlib.sha256()
    deps = [os.path.join(_HERE, "csrc", s) for s in _SOURCES]
    deps.append(os.path.join(os.path.dirname(_HERE), "include", "sdv.h"))
    for d in deps:
        with open(d, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def _stale() -> bool:
    if not os.path.exists(LIB_PATH) or not os.path.exists(HASH_PATH):
        return True
    with open(HASH_PATH) as fh:
        return fh.read().strip() != _source_hash()


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-Xcompiler", "-fPIC"]
    if verbose:
        flags[1:1] = ["-Xptxas", "-v"]
    objects = [os.path.join(_HERE, "csrc", u[:-3] + ".o") for u in _UNITS]
    commands = [flags + ["-c", "-o", o, os.path.join(_HERE, "csrc", u)] for u, o in zip(_UNITS, objects)]
    if verbose:
        print("\n".join(" ".join(c) for c in commands))
    running = [subprocess.Popen(c) for c in commands]
    for p, c in [(p, p.wait()) for p in running]:
        if c:
            raise subprocess.CalledProcessError(c, p.args)
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB_PATH + ".tmp"] + objects, check=True)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    with open(HASH_PATH, "w") as fh:
        fh.write(_source_hash())
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
