"""Build the C-ABI CUDA library in-tree for sm_100a (nvcc cross-compiles without a GPU) and the Python call module beside it."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblrbi.so")
SOURCES = ["api.cu", "decode_kernels.cu", "gemv_kernels.cu", "gemm_tc.cu", "alg1_kernels.cu", "ranked_kernels.cu", "backward_kernels.cu", "nmf_kernels.cu",
           "norm_forward.cu", "norm_backward.cu", "keep_kernels.cu", "w4_kernels.cu", "api_block.cu"]
CALLS = os.path.join(HERE, "_lrbi_torch.so")
CALLS_SOURCE = os.path.join(CSRC, "torch_calls.cpp")


def _stale(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    header = os.path.join(ROOT, "include", "lrbi.h")
    kernels = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))]
    if force or _stale(LIB, kernels + [header]):
        _build_library(verbose)
    if force or _stale(CALLS, [CALLS_SOURCE, header]):
        _build_calls()
    return LIB


def _build_calls() -> None:
    """The Python module that marshals torch tensors into the C ABI's calls."""
    import importlib.util
    import sysconfig

    torch_dir = importlib.util.find_spec("torch").submodule_search_locations[0]
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    tmp = CALLS + ".tmp.%d" % os.getpid()
    include = [os.path.join(ROOT, "include"), os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-w"]
    cmd += ["-I" + d for d in include] + [CALLS_SOURCE, "-o", tmp, "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]
    cmd += ["-L" + os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, CALLS)


def _build_library(verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [
        nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
        "-shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    ]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES] + ["-o", tmp]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
