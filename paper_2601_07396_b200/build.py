"""Builds, in-tree, ``libsvdcache.so`` (the C-ABI CUDA library) with nvcc for sm_100a, and ``_calls.*.so`` (the argument side
of the 8-bit calls, a Python extension over torch's tensors) with the host compiler.  The library needs neither the other
nor torch."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsvdcache.so")
CALLS_SOURCE = os.path.join(CSRC, "calls.cpp")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--expt-relaxed-constexpr",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def calls_path() -> str:
    """The extension for this interpreter and this torch: its name says both, so that one built with others is not loaded."""
    import torch
    return os.path.join(HERE, f"_calls.{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}.so")


def build_calls(force: bool = False) -> str:
    """Compile csrc/calls.cpp into the extension.  Returns its path."""
    path = calls_path()
    deps = [CALLS_SOURCE, os.path.join(HERE, "..", "include", "svdcache.h")]
    if not force and os.path.exists(path) and all(os.path.getmtime(d) <= os.path.getmtime(path) for d in deps):
        return path
    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [sysconfig.get_paths()["include"], *cpp_extension.include_paths(), os.path.join(cuda, "include")]
    lib_dir = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = path + f".tmp{os.getpid()}"
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
                    f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[a for d in include for a in ("-isystem", d)],
                    CALLS_SOURCE, "-o", tmp, f"-L{lib_dir}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"], check=True)
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into one shared object.  Returns its path."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    procs = []
    build_dir = os.path.join(HERE, "_build")
    os.makedirs(build_dir, exist_ok=True)
    for src in sources():
        obj = os.path.join(build_dir, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd)))
        objs.append(obj)
    for src, p in procs:
        if p.wait() != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp, *objs], check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_calls(force="--force" in sys.argv))
