"""Build the C-ABI CUDA library in-tree for sm_100a (nvcc cross-compiles without a GPU) and the Python call module beside it."""
from __future__ import annotations

import importlib.util
import os
import re
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblrbi.so")
SOURCES = ["api.cu", "decode_kernels.cu", "gemv_kernels.cu", "gemm_tc.cu", "alg1_kernels.cu", "ranked_kernels.cu", "backward_kernels.cu", "nmf_kernels.cu",
           "norm_forward.cu", "norm_backward.cu", "keep_kernels.cu", "w4_kernels.cu", "api_block.cu"]
CALLS_SOURCE = os.path.join(CSRC, "torch_calls.cpp")


def _torch_dir() -> str | None:
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec else None


def torch_version() -> str | None:
    """Version of the installed torch (without importing it), or None."""
    where = _torch_dir()
    if where is None:
        return None
    with open(os.path.join(where, "version.py")) as f:
        found = re.search(r"^__version__ = ['\"](.+)['\"]", f.read(), re.M)
    return found.group(1) if found else "unknown"


def calls_path() -> str | None:
    """The call module of the installed torch: it depends on the C++ ABI of that version, and on the interpreter's."""
    version = torch_version()
    return version and os.path.join(HERE, "_lrbi_torch-%s%s" % (version, sysconfig.get_config_var("EXT_SUFFIX")))


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
    calls = calls_path()
    if calls is None:
        print("torch is not installed: %s is complete, the Python call module was not built" % os.path.basename(LIB), file=sys.stderr)
    elif force or _stale(calls, [CALLS_SOURCE, header]):
        _build_calls(calls)
    return LIB


def _build_calls(target: str) -> None:
    """The Python module that marshals torch tensors into the C ABI's calls."""
    torch_dir = _torch_dir()
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    tmp = target + ".tmp.%d" % os.getpid()
    include = [os.path.join(ROOT, "include"), os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-w"]
    cmd += ["-I" + d for d in include] + [CALLS_SOURCE, "-o", tmp, "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]
    cmd += ["-L" + os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, target)


def _build_library(verbose: bool) -> None:
    """An nvcc a source, as many at a time as there are processors: one after the other they take more than twice as long."""
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    flags = arch + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    tmp = LIB + ".tmp.%d" % os.getpid()
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(os.cpu_count()) as pool:
        def compiled(source):
            out = os.path.join(objects, source[:-3] + ".o")
            subprocess.run([nvcc, *flags, "-c", os.path.join(CSRC, source), "-o", out], check=True)
            return out

        # the longest first
        order = sorted(SOURCES, key=lambda f: -os.path.getsize(os.path.join(CSRC, f)))
        subprocess.run([nvcc, *arch, "-shared", *pool.map(compiled, order), "-o", tmp], check=True)
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
