"""Builds libsr_rollout.so (the C-ABI library) in-tree with nvcc for sm_100a, and the Python extension of its operators."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsr_rollout.so")
EXTENSION = os.path.join(HERE, "_operators.so")         # the operators' calls from Python (csrc/sr_python.cpp)
SOURCES = ["sr_compile.cpp", "sr_api.cu", "sr_input.cu", "sr_direct.cu", "sr_tc.cu", "sr_resident.cu", "sr_dense.cu",
           "sr_norm.cu", "sr_product.cu", "sr_memory.cu", "sr_chunks.cu"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-cudart", "static"]


EXTENSION_SOURCE = "sr_python.cpp"


def _stale(built: str, sources) -> bool:
    if not os.path.exists(built):
        return True
    t = os.path.getmtime(built)
    deps = [os.path.join(CSRC, f) for f in sources] + [os.path.join(HERE, "..", "include", "sr_rollout.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """The library, which needs nvcc only, and the operators' extension, which needs PyTorch, a host compiler and Python's headers: where one of these is missing
    there is a warning, and importing the operators says why it fails."""
    build_library(force, verbose)
    if force or _stale(EXTENSION, [EXTENSION_SOURCE]):
        try:
            build_extension()
        except (ImportError, OSError, subprocess.CalledProcessError) as e:
            import warnings
            warnings.warn("the operators' extension is not built: %s" % e)
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale(LIB, [f for f in os.listdir(CSRC) if f != EXTENSION_SOURCE]):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(objdir, src + ".o")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-x", "cu", "-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError("nvcc failed on %s" % src)
    tmp = LIB + ".%d.tmp" % os.getpid()
    subprocess.check_call([nvcc, "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a",
                           "-o", tmp] + objs)
    os.replace(tmp, LIB)
    return LIB


def build_extension() -> str:
    """Compiles the CPython extension against the installed PyTorch; it finds the library beside it."""
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    include = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"), "/usr/local/cuda/include",
               sysconfig.get_paths()["include"]]
    tmp = EXTENSION + ".%d.tmp" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
                           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI] + ["-I" + i for i in include] +
                          [os.path.join(CSRC, EXTENSION_SOURCE), "-o", tmp, "-L" + HERE, "-l:libsr_rollout.so", "-L" + os.path.join(base, "lib"), "-ltorch_python", "-ltorch",
                           "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + os.path.join(base, "lib")])
    os.replace(tmp, EXTENSION)
    return EXTENSION


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
