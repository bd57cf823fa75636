"""Builds libspd.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libspd.so")
SOURCES = ["spd_kernel.cu", "spd_prefill.cu", "spd_prefill_tc.cu", "spd_batch.cu", "spd_api.cu", "spd_ngram.cu",
           "spd_append.cu", "spd_attend.cu", "spd_attend_bf16.cu", "spd_attend_terms.cu", "spd_attend_few.cu", "spd_attend_few_float.cu", "spd_attend_eight.cu", "spd_attend_float.cu", "spd_select.cu",
           "spd_reorder.cu"]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: libspd.so cannot be built")
    return exe


def tensors_path() -> str:
    """The module that takes torch tensors to the beams' operators: a file of its own for each Python and torch, whose layouts are compiled into it."""
    import torch

    return os.path.join(HERE, "_spd_tensors-%s-torch%s.so" % (sysconfig.get_config_var("SOABI"), torch.__version__))


def _stale(target: str = LIB) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    own = "spd_tensors.cpp"
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if (f == own) == (target != LIB)] + [os.path.join(INCLUDE, "spd.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_tensors(force: bool = False) -> str:
    """Builds the module that takes torch tensors to the operators (a C++ compiler and torch's headers, no GPU code)."""
    target = tensors_path()
    if not force and not _stale(target):
        return target
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths

    tmp = target + ".tmp%d" % os.getpid()
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, "-I", INCLUDE]
    for path in [*include_paths(), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", path]
    cmd += ["-o", tmp, os.path.join(CSRC, "spd_tensors.cpp")]
    for path in library_paths():
        cmd += ["-L", path]
    subprocess.check_call(cmd + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch", "-ltorch_python"])
    os.replace(tmp, target)
    return target


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    with tempfile.TemporaryDirectory() as work:                       # the sources side by side, then the library
        def compile_one(source: str) -> str:
            obj = os.path.join(work, source + ".o")
            subprocess.check_call([_nvcc(), *flags, "-c", "-o", obj, os.path.join(CSRC, source)])
            return obj

        with ThreadPoolExecutor(max_workers=max(1, min(len(SOURCES), os.cpu_count() or 1))) as pool:
            objects = list(pool.map(compile_one, SOURCES))
        subprocess.check_call([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC", "-o", tmp, *objects])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
    print(build_tensors())
