"""Build libproxyformer.so (the sm_103a CUDA library) in-tree with nvcc.

Each .cu file under csrc/ compiles to an object in parallel, then one shared
library is linked next to this file, and the native part of local.py
(csrc/local_binding.cpp, _local.so) against it.  Usage: ``python -m
paper_2608_23463_gb300.buildlib`` or ``build()`` from Python.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libproxyformer.so")
BINDING = os.path.join(HERE, "_local.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _nvcc() -> str:
    cand = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found (set NVCC or put CUDA's bin on PATH)")
    return cand


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def binding_tag() -> str:
    """Interpreter and torch that local_binding.cpp is compiled for: its object's name and its
    module's ``built_for`` hold them, so that an upgrade of either takes effect."""
    import torch
    return f"{sys.implementation.cache_tag}-torch-{torch.__version__}"


def binding_object() -> str:
    return os.path.join(OUT_DIR, f"local_binding.{binding_tag()}.o")


def _compile_binding(obj: str) -> None:
    """local_binding.cpp against the headers of the installed torch."""
    import sysconfig

    import torch
    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    dirs = [os.path.join(ROOT, "include"), inc, os.path.join(inc, "torch", "csrc", "api", "include"),
            sysconfig.get_paths()["include"], cuda]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DPF_BUILT_FOR="{binding_tag()}"',
           *(f"-I{d}" for d in dirs), "-c", os.path.join(CSRC, "local_binding.cpp"), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed on local_binding.cpp:\n{r.stdout}\n{r.stderr}")


def _link_binding(obj: str) -> None:
    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = [os.environ.get("CXX", "g++"), "-shared", obj, "-o", BINDING + ".tmp", f"-L{HERE}",
           "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN", f"-L{lib}", "-lc10", "-lc10_cuda",
           "-ltorch_cpu", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"linking {BINDING} failed:\n{r.stdout}\n{r.stderr}")
    os.replace(BINDING + ".tmp", BINDING)


def build(verbose: bool = False, extra_flags=()) -> str:
    nvcc = _nvcc()
    os.makedirs(OUT_DIR, exist_ok=True)
    srcs = _sources()
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    deps.append(os.path.join(ROOT, "include", "proxyformer.h"))
    newest_dep = max(os.path.getmtime(p) for p in deps)

    def compile_one(src):
        obj = os.path.join(OUT_DIR, os.path.basename(src)[:-3] + ".o")
        if (os.path.exists(obj) and os.path.getmtime(obj) >= os.path.getmtime(src)
                and os.path.getmtime(obj) >= newest_dep and not extra_flags):
            return obj
        cmd = [nvcc, *ARCH, *FLAGS, *extra_flags, "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr, file=sys.stderr)
        return obj

    bind_src, bind_obj = os.path.join(CSRC, "local_binding.cpp"), binding_object()
    bind_deps = max(os.path.getmtime(bind_src), os.path.getmtime(deps[-1]))

    with ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as ex:
        stale = not os.path.exists(bind_obj) or os.path.getmtime(bind_obj) < bind_deps
        binding = ex.submit(_compile_binding, bind_obj) if stale else None
        objs = list(ex.map(compile_one, srcs))
        if binding is not None:
            binding.result()
    cmd = [nvcc, *ARCH, "-shared", "-Xlinker", "-soname=" + os.path.basename(LIB), "-o", LIB + ".tmp",
           *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(LIB + ".tmp", LIB)
    _link_binding(bind_obj)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
