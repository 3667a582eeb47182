"""Compile the CUDA sources under csrc/ into librptq.so (sm_100a only), and calls.cpp, which hands PyTorch's tensors to it, into _calls.so; in-tree."""
from __future__ import annotations

import glob
import importlib.util
import os
import subprocess
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


def needs_build() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(CALLS):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALLS))
    return any(os.path.getmtime(d) > t for d in dependencies())


def build_calls() -> str:
    """calls.cpp against the headers of the installed PyTorch; it finds librptq.so beside itself."""
    torch = os.path.join(importlib.util.find_spec("torch").submodule_search_locations[0])
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    tmp = CALLS + f".tmp{os.getpid()}"
    subprocess.run(["g++", "-shared", "-fPIC", "-O2", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
                    "-I", os.path.join(torch, "include"), "-I", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                    "-I", os.path.join(cuda, "include"), os.path.join(CSRC, "calls.cpp"), "-o", tmp, "-L", HERE, "-l:librptq.so", "-Wl,-rpath,$ORIGIN",
                    "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"], check=True)
    os.replace(tmp, CALLS)
    return CALLS


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = ["nvcc", "-shared", "--threads", str(os.cpu_count() or 1), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
           *sources(), "-o", tmp, "-lgomp"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    build_calls()
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
