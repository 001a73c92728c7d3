"""Build libntc.so (CUDA for sm_103a) in-tree, with nvcc only.

Each .cu file under csrc/ compiles to an object in parallel; the objects link
into ``_build/libntc.so`` with the CUDA runtime linked statically, so the
library needs nothing but the driver at run time.  Beside it g++ compiles
``_build/_experts.so``, the torch binding of the routed-expert calls
(csrc/torch/), against the installed torch's headers; without torch it is left out,
for the library does not need it.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libntc.so")
BINDING = os.path.join(BUILD, "_experts.so")
BINDING_SOURCE = os.path.join(CSRC, "torch", "experts_binding.cpp")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I", INCLUDE]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.exists(c) or c == "nvcc"):
            return c
    raise RuntimeError("nvcc not found")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")
    return r.stdout + r.stderr


def _binding_object() -> str | None:
    import sysconfig

    try:
        import torch
    except ImportError:
        return None
    t = os.path.join(os.path.dirname(torch.__file__), "include")
    obj = os.path.join(BUILD, f"experts_binding.{torch.__version__}.o")
    if _stale(obj, [BINDING_SOURCE, os.path.join(INCLUDE, "ntc.h")]):
        cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include")
        _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE, "-isystem", t, "-isystem",
              os.path.join(t, "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"],
              "-isystem", cuda, "-c", BINDING_SOURCE, "-o", obj], f"g++ on {BINDING_SOURCE}")
    return obj


def _link_binding(obj: str) -> None:
    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    if _stale(BINDING, [obj, LIB]):
        tmp = BINDING + f".tmp{os.getpid()}"
        _run(["g++", "-shared", "-o", tmp, obj, LIB, "-L", lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10",
              "-lc10_cuda", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{lib}"], "link of the torch binding")
        os.replace(tmp, BINDING)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + [os.path.join(INCLUDE, "ntc.h")]
    nvcc = _nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        if force or ptxas_info or _stale(obj, [src] + headers):
            cmd = [nvcc, *ARCH, *FLAGS, "-c", src, "-o", obj]
            if ptxas_info:
                cmd.insert(1, "-Xptxas=-v")
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
            if verbose or ptxas_info:
                sys.stderr.write(r.stdout + r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(sources))) as ex:
        binding = ex.submit(_binding_object)
        objs = list(ex.map(compile_one, sources))
        binding = binding.result()
    if force or _stale(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        _run([nvcc, *ARCH, "-shared", "-cudart", "static", "-Xlinker", "-soname=libntc.so", "-o", tmp, *objs], "link")
        os.replace(tmp, LIB)
    if binding:
        _link_binding(binding)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, ptxas_info="--ptxas" in sys.argv))
