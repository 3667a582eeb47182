"""Compile the CUDA sources under csrc/ into librptq.so (sm_100a only), and calls.cpp, which hands PyTorch's tensors to it, into _calls.so; in-tree.

librptq.so needs nvcc alone. _calls.so is built where a PyTorch for CUDA is installed, for that PyTorch and Python: without it `binding.KvCache`
raises, everything else works."""
from __future__ import annotations

import glob
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librptq.so")
CALLS = os.path.join(HERE, "_calls.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC,-fopenmp,-ffp-contract=off,-fno-fast-math,-Wall",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def dependencies():
    headers = [os.path.join(CSRC, "*.h"), os.path.join(CSRC, "*.cuh"), os.path.join(CSRC, "*.cpp"), os.path.join(ROOT, "include", "*.h")]
    return sources() + [f for pattern in headers for f in sorted(glob.glob(pattern))]


def _older(target: str, files) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(f) > os.path.getmtime(target) for f in files)


def _torch():
    """The installed PyTorch's folder; None if there is none, or one without CUDA."""
    spec = importlib.util.find_spec("torch")
    at = spec.submodule_search_locations[0] if spec and spec.submodule_search_locations else None
    return at if at and os.path.exists(os.path.join(at, "lib", "libc10_cuda.so")) else None


def _calls_tag() -> str:
    """What _calls.so is built for; it carries this text."""
    try:
        torch = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:                         # built from source, without an installation's record
        torch = _torch()
    return f"rptq calls for torch {torch}, {sys.implementation.cache_tag};"


def library_is_stale() -> bool:
    return _older(LIB, [f for f in dependencies() if not f.endswith(".cpp")])


def calls_are_stale() -> bool:
    if _torch() is None:
        return False
    if _older(CALLS, [os.path.join(CSRC, "calls.cpp"), os.path.join(ROOT, "include", "rptq.h")]):
        return True
    with open(CALLS, "rb") as f:
        return _calls_tag().encode() not in f.read()


def needs_build() -> bool:
    return library_is_stale() or calls_are_stale()


def build_calls() -> str:
    """calls.cpp against the headers of the installed PyTorch; it finds librptq.so beside itself."""
    torch = _torch()
    cuda = os.environ.get("CUDA_HOME") or os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")))
    tmp = CALLS + f".tmp{os.getpid()}"
    subprocess.run(["g++", "-shared", "-fPIC", "-O2", "-std=c++17", "-Wall", f'-DRPTQ_CALLS_TAG="{_calls_tag()}"',
                    "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
                    "-I", os.path.join(torch, "include"), "-I", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                    "-I", os.path.join(cuda, "include"), os.path.join(CSRC, "calls.cpp"), "-o", tmp, "-L", HERE, "-l:librptq.so", "-Wl,-rpath,$ORIGIN",
                    "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"], check=True)
    os.replace(tmp, CALLS)
    return CALLS


def build(force: bool = False, verbose: bool = False) -> str:
    if force or library_is_stale():
        tmp = LIB + f".tmp{os.getpid()}"
        cmd = ["nvcc", "-shared", "--threads", str(os.cpu_count() or 1), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
               *sources(), "-o", tmp, "-lgomp"]
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    if calls_are_stale() or (force and _torch() is not None):
        build_calls()
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
