"""Build the CUDA library libsss.so in-tree with nvcc (sm_103a only), and with g++
_binding.so, the compiled part of the Python binding.  The library needs nvcc alone;
the binding is built apart from it, for the torch and Python that will load it.

Each translation unit under csrc/ is compiled in parallel to an object file
under _build/, then linked into paper_2607_08779_gb300/libsss.so.  The CUDA
runtime is linked statically; the driver entry point needed for tensor maps
is resolved at run time, so the library loads on machines without a GPU.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libsss.so")
BINDING_SRC = os.path.join(CSRC, "binding.cpp")
BINDING = os.path.join(PKG, "_binding.so")
STAMP = os.path.join(BUILD, "binding.stamp")  # what _binding.so was built for

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
              "--expt-relaxed-constexpr", "-I", INCLUDE, "-I", CSRC]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libsss.so")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    files = sources() + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")]
    return files + _common_deps()


def _common_deps():
    return [os.path.join(INCLUDE, "sss.h"), os.path.abspath(__file__)]


def _newer(target, files) -> bool:
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(f) <= t for f in files)


def up_to_date() -> bool:
    return _newer(LIB, _deps())


def _stamp() -> str:
    import platform
    import sys

    import torch

    return "\n".join((torch.__version__, torch.__file__, sys.version, platform.machine()))


def binding_up_to_date() -> bool:
    """Whether _binding.so is there, newer than its sources, and built for this
    interpreter and the torch that it imports."""
    if not _newer(BINDING, [BINDING_SRC] + _common_deps()) or not os.path.exists(STAMP):
        return False
    with open(STAMP) as f:
        return f.read() == _stamp()


def build_binding(force: bool = False) -> str:
    """_binding.so, against the torch that this interpreter imports."""
    import sysconfig

    import torch

    if not force and binding_up_to_date():
        return BINDING
    os.makedirs(BUILD, exist_ok=True)
    home = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    include = [INCLUDE, os.path.join(home, "include"),
               os.path.join(home, "include", "torch", "csrc", "api", "include"), cuda,
               sysconfig.get_paths()["include"]]
    tmp = BINDING + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[x for d in include for x in ("-isystem", d)], BINDING_SRC, "-o", tmp,
           "-L", os.path.join(home, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python",
           f"-Wl,-rpath,{os.path.join(home, 'lib')}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for {BINDING_SRC}:\n{r.stderr}")
    os.replace(tmp, BINDING)
    tmp = STAMP + f".tmp{os.getpid()}"
    with open(tmp, "w") as f:
        f.write(_stamp())
    os.replace(tmp, STAMP)
    return BINDING


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    cc = nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        cmd = [cc, *ARCH, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr)
        return obj

    srcs = sources()
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs), os.cpu_count() or 4)) as ex:
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [cc, *ARCH, "-shared", "-Xcompiler", "-fPIC", "-o", tmp, *objs,
           "-cudart", "static"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys

    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv,
                extra_flags=["-Xptxas", "-v"] if "--ptxas" in sys.argv else ()))
