"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU), and beside it the module that calls it on torch tensors.  The two are kept
apart: the library depends on neither torch nor Python, and neither is rebuilt, nor missed, because of the other."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsdv.so")
TORCH_PATH = os.path.join(_HERE, "_paged.so")   # paged.py's calls on torch tensors
_UNITS = ["sdv.cu", "paged.cu"]   # compiled side by side
_SOURCES = _UNITS + ["forward.cuh", "dense.cuh", "device_once.h", "layout.cuh", "overlap.h", "paged.cuh", "ptx.cuh", "small_gemm.cuh", "small_kernels.cuh",
                     "tensor_map.h", "tree_attention.cuh", "tree_plan.h", "verify_sampled.cuh"]
_TORCH_SOURCES = ["paged_torch.cpp"]


def _digest(sources, what: str = "") -> str:
    """Digest of sources and the header (file times do not survive a checkout or a copy)."""
    import hashlib
    h = hashlib.sha256(what.encode())
    for d in [os.path.join(_HERE, "csrc", s) for s in sources] + [os.path.join(os.path.dirname(_HERE), "include", "sdv.h")]:
        with open(d, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def _torch_digest() -> str:
    import sys
    import torch
    return _digest(_TORCH_SOURCES, f"torch {torch.__version__} python {sys.version}")


def _stale(path: str, digest: str) -> bool:
    if not os.path.exists(path) or not os.path.exists(path + ".srchash"):
        return True
    with open(path + ".srchash") as fh:
        return fh.read().strip() != digest


def _done(path: str, digest: str) -> str:
    os.replace(path + ".tmp", path)
    with open(path + ".srchash", "w") as fh:
        fh.write(digest)
    return path


def _start(commands, verbose: bool):
    if verbose:
        print("\n".join(" ".join(c) for c in commands))
    return [subprocess.Popen(c) for c in commands]


def _wait(running) -> None:
    for p, c in [(p, p.wait()) for p in running]:
        if c:
            raise subprocess.CalledProcessError(c, p.args)


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


def build_library(force: bool = False, verbose: bool = False) -> str:
    """The library alone, if its sources are newer."""
    digest = _digest(_SOURCES)
    if not force and not _stale(LIB_PATH, digest):
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-Xcompiler", "-fPIC"]
    if verbose:
        flags[1:1] = ["-Xptxas", "-v"]
    objects = [os.path.join(_HERE, "csrc", u[:-3] + ".o") for u in _UNITS]
    _wait(_start([flags + ["-c", "-o", o, os.path.join(_HERE, "csrc", u)] for u, o in zip(_UNITS, objects)], verbose))
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB_PATH + ".tmp"] + objects, check=True)
    return _done(LIB_PATH, digest)


def build_torch_calls(force: bool = False, verbose: bool = False) -> str:
    """The module of paged.py alone, if its source, torch or Python is another."""
    digest = _torch_digest()
    if not force and not _stale(TORCH_PATH, digest):
        return TORCH_PATH
    _wait(_start([_torch_command(TORCH_PATH + ".tmp")], verbose))
    return _done(TORCH_PATH, digest)


def build(force: bool = False, verbose: bool = False) -> str:
    """Both, side by side.  What fails of one is raised behind the other."""
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(1) as pool:
        calls = pool.submit(build_torch_calls, force, verbose)
        library = build_library(force, verbose)
        calls.result()
    return library


if __name__ == "__main__":
    print(build(force=True, verbose=True))
