"""Compile the HIP libraries for gfx950 with hipcc, and the PyTorch binding.

All HIP sources under ``csrc/`` are compiled into one shared library,
``librcdp.so``, next to this file: the solver behind include/rc.h.  The
microbenchmarks of the chip's peaks under ``peak/`` (measurement only, not
part of the solver) go into ``libpeak.so``.  Packed-FP32 instruction
selection is disabled.  The operators' PyTorch binding under ``bind/`` is
host code: g++ compiles it against the installed PyTorch into ``_ops.so``.
"""

import glob
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "librcdp.so")
OPS_LIB = os.path.join(HERE, "_ops.so")
PEAK_LIB = os.path.join(HERE, "libpeak.so")
ARCH = os.environ.get("RCDP_OFFLOAD_ARCH", "gfx950")


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))


OBJ_DIR = os.path.join(ROOT, "_build")
FLAGS = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]


def command(out, srcs=None):
    """One hipcc line that builds the shared library from the sources."""
    return ["hipcc"] + FLAGS + ["-shared"] + (sources() if srcs is None else srcs) + ["-o", out]


def _compile(lib, srcs, verbose):
    """Each source to an object (in parallel), then one shared library."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs = [os.path.join(OBJ_DIR, os.path.basename(src) + ".o") for src in srcs]

    def one(pair):
        src, obj = pair
        cmd = ["hipcc"] + FLAGS + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)

    jobs = max(1, min(len(srcs), int(os.environ.get("MAX_JOBS", os.cpu_count() or 4))))
    with ThreadPoolExecutor(jobs) as pool:
        list(pool.map(one, zip(srcs, objs)))
    tmp = lib + ".tmp"
    cmd = ["hipcc", f"--offload-arch={ARCH}", "-shared", "-fPIC"] + objs + ["-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, lib)


def bind_command(out):
    """One g++ line that builds the PyTorch binding (links librcdp.so)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    include = [os.path.join(ROOT, "include"), *cpp_extension.include_paths(),
               os.path.join(rocm, "include"), sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
             "-DUSE_ROCM=1", "-DTORCH_EXTENSION_NAME=_ops",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
            + [x for d in include for x in ("-isystem", d)]
            + [os.path.join(HERE, "bind", "ops_bind.cpp"), "-L", HERE, "-lrcdp", "-L", lib, "-lc10",
               "-lc10_hip", "-ltorch_cpu", "-ltorch", "-ltorch_python", "-Wl,-rpath,$ORIGIN", "-o", out])


def build_binding(verbose=False):
    cmd = bind_command(OPS_LIB + ".tmp")
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(OPS_LIB + ".tmp", OPS_LIB)


def build(verbose=False):
    _compile(LIB, sources(), verbose)
    build_binding(verbose)
    _compile(PEAK_LIB, sorted(glob.glob(os.path.join(HERE, "peak", "*.hip"))), verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
