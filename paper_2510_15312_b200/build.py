"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU), and beside it the module that calls it on torch tensors."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsdv.so")
TORCH_PATH = os.path.join(_HERE, "_paged.so")   # paged.py's calls on torch tensors
_UNITS = ["sdv.cu", "paged.cu"]   # compiled side by side
_SOURCES = _UNITS + ["forward.cuh", "dense.cuh", "device_once.h", "layout.cuh", "overlap.h", "paged.cuh", "ptx.cuh", "small_gemm.cuh", "small_kernels.cuh",
                     "paged_torch.cpp", "tensor_map.h", "tree_attention.cuh", "tree_plan.h", "verify_sampled.cuh"]


HASH_PATH = LIB_PATH + ".srchash"


def _source_hash() -> str:
    """Digest of every source the library is built from (file times do not survive a checkout or a copy)."""
    import hashlib
    import sys
    import torch
    h = hashlib.sha256(f"torch {torch.__version__} python {sys.version}".encode())
    deps = [os.path.join(_HERE, "csrc", s) for s in _SOURCES]
    deps.append(os.path.join(os.path.dirname(_HERE), "include", "sdv.h"))
    for d in deps:
        with open(d, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def _stale() -> bool:
    if not all(os.path.exists(p) for p in (LIB_PATH, TORCH_PATH, HASH_PATH)):
        return True
    with open(HASH_PATH) as fh:
        return fh.read().strip() != _source_hash()


def _torch_command(out: str):
    """Compiles csrc/paged_torch.cpp against the installed torch (host code only)."""
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}"]
    for i in includes:
        cmd += ["-isystem", i]
    lib = os.path.join(root, "lib")
    return cmd + ["-o", out, os.path.join(_HERE, "csrc", "paged_torch.cpp"), "-L" + lib, "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath," + lib]


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-Xcompiler", "-fPIC"]
    if verbose:
        flags[1:1] = ["-Xptxas", "-v"]
    objects = [os.path.join(_HERE, "csrc", u[:-3] + ".o") for u in _UNITS]
    commands = [flags + ["-c", "-o", o, os.path.join(_HERE, "csrc", u)] for u, o in zip(_UNITS, objects)]
    commands.append(_torch_command(TORCH_PATH + ".tmp"))
    if verbose:
        print("\n".join(" ".join(c) for c in commands))
    running = [subprocess.Popen(c) for c in commands]
    for p, c in [(p, p.wait()) for p in running]:
        if c:
            raise subprocess.CalledProcessError(c, p.args)
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB_PATH + ".tmp"] + objects, check=True)
    os.replace(TORCH_PATH + ".tmp", TORCH_PATH)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    with open(HASH_PATH, "w") as fh:
        fh.write(_source_hash())
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
