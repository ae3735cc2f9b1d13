"""Builds libbcp.so (host planner + sm_100a kernels + C ABI) in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libbcp.so")
SOURCES = ["planner.cpp", "units.cpp", "api.cu", "plan_image.cu", "host_path.cu", "kernels.cu", "tma_kernel.cu", "convert_kernel.cu", "static_pack.cu", "stager.cu", "export.cu", "ipc.cu",
           "rope.cu", "kv_cache.cu", "kv_attend.cu", "kv_prefix.cu", "verify.cu"]
HEADERS = ["plan.hpp", "kernels.cuh", "host_threads.hpp", "plan_object.hpp", "tma_ptx.cuh", "copy_loops.cuh", "decode.cuh", "attend.cuh"]


BINDING = os.path.join(CSRC, "binding.cpp")


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; libbcp.so cannot be built")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(INCLUDE, "bcp.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile for sm_100a only; returns the path of the shared library."""
    if not force and not is_stale():
        return LIB
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC,-fvisibility=hidden"]

    def nvcc(*args):
        cmd = [nvcc_path(), *flags, *args]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
        if verbose:
            sys.stderr.write(r.stdout + r.stderr)

    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, f + ".o") for f in SOURCES]
        more = ["-Xptxas", "-v"] if verbose else []
        with ThreadPoolExecutor(os.cpu_count()) as pool:  # the kernels take most of the time: a process for each file
            for done in [pool.submit(nvcc, *more, "-c", "-I", INCLUDE, "-I", CSRC, os.path.join(CSRC, f), "-o", o) for f, o in zip(SOURCES, objects)]:
                done.result()
        nvcc("-shared", *objects, "-o", LIB, *(["-lcuda"] if os.environ.get("BCP_LINK_DRIVER") else []))
    return LIB


def binding_path() -> str:
    """The module that takes torch tensors: one file per torch and Python version, whose headers it was built with."""
    import torch

    tag = "".join(c if c.isalnum() else "_" for c in f"{torch.__version__}_py{sys.version_info[0]}{sys.version_info[1]}")
    return os.path.join(HERE, f"_binding_{tag}.so")


def build_binding(force: bool = False) -> str:
    """Compile csrc/binding.cpp against the installed torch, if there is no newer module; returns its path."""
    import sysconfig

    import torch

    path = binding_path()
    if not force and os.path.exists(path) and all(os.path.getmtime(d) <= os.path.getmtime(path) for d in (BINDING, os.path.join(INCLUDE, "bcp.h"))):
        return path
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(nvcc_path()))
    include = [INCLUDE, os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX") or shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for d in include:
        cmd += ["-isystem" if d != INCLUDE else "-I", d]
    partial = f"{path}.{os.getpid()}"
    cmd += [BINDING, "-o", partial, "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("the binding does not compile:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    os.replace(partial, path)
    return path


def build_all(force: bool = False, verbose: bool = False) -> list:
    """The library and, where torch is installed, the module that takes its tensors (the decoding operators)."""
    import importlib.util

    paths = [build_library(force=force, verbose=verbose)]
    if importlib.util.find_spec("torch") is not None:
        paths.append(build_binding(force=force))
    return paths


if __name__ == "__main__":
    print("\n".join(build_all(force=True, verbose="-v" in sys.argv)))
