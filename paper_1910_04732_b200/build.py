"""Builds the CUDA library in-tree, csrc/flop_lib.cu and csrc/flop_rows.cu -> libflop_b200.so (sm_100a only), and the native half of the Python
binding, csrc/binding_native.cpp -> _binding_native.<python and torch it is for>.so."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
UNITS = [os.path.join(HERE, "csrc", f) for f in ("flop_lib.cu", "flop_rows.cu")]
ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]
OBJECTS = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libflop_b200.so")
NATIVE_SRC = os.path.join(HERE, "csrc", "binding_native.cpp")


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    d = os.path.join(HERE, "csrc")
    inc = os.path.join(os.path.dirname(HERE), "include", "flop.h")
    return [os.path.join(d, f) for f in sorted(os.listdir(d)) if f.endswith((".cu", ".cuh", ".h"))] + [inc]


def _includes(path, seen=None):
    """`path` and the files of this repository that it includes, directly or not."""
    seen = set() if seen is None else seen
    path = os.path.normpath(path)
    if path not in seen and os.path.exists(path):
        seen.add(path)
        with open(path) as f:
            for name in re.findall(r'^#include "([^"]+)"', f.read(), re.M):
                _includes(os.path.join(os.path.dirname(path), name), seen)
    return seen


def up_to_date() -> bool:
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(s) <= t for s in sources())


def native_path() -> str:
    """The module is bound to the C++ interface of one torch and one Python: its name carries both, so that no other loads it."""
    import torch
    return os.path.join(HERE, f"_binding_native.{sys.implementation.cache_tag}-torch-{torch.__version__}.so")


def native_up_to_date() -> bool:
    path = native_path()
    if not os.path.exists(path):
        return False
    t = os.path.getmtime(path)
    return all(os.path.getmtime(p) <= t for p in (NATIVE_SRC, sources()[-1]))


def build_native(force: bool = False) -> str:
    """The module links to libflop_b200.so beside it and to the torch libraries that `import torch` has loaded."""
    path = native_path()
    if not force and native_up_to_date():
        return path
    import torch
    t = os.path.dirname(os.path.abspath(torch.__file__))
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I" + os.path.join(t, "include"), "-I" + os.path.join(t, "include", "torch", "csrc", "api", "include"),
           "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(cuda, "include"), "-o", path, NATIVE_SRC,
           "-L" + os.path.join(t, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-L" + HERE, "-l:libflop_b200.so",
           "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("building the native binding failed:\n" + r.stdout + r.stderr)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and up_to_date():
        build_native()
        return LIB
    os.makedirs(OBJECTS, exist_ok=True)
    jobs, objects = [], []
    for unit in UNITS:                     # the units compile side by side; one whose sources are older than its object is kept
        obj = os.path.join(OBJECTS, os.path.basename(unit) + ".o")
        objects.append(obj)
        if not force and not verbose and os.path.exists(obj) and all(os.path.getmtime(p) <= os.path.getmtime(obj) for p in _includes(unit)):
            continue
        cmd = [_nvcc(), *(["-Xptxas", "-v"] if verbose else []), *ARCH, "-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-c", "-o", obj, unit]
        jobs.append((obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = ""
    for obj, job in jobs:
        out, _ = job.communicate()
        if job.returncode != 0:
            failed += out
            if os.path.exists(obj):
                os.remove(obj)
        elif verbose:
            print(out)
    if failed:
        raise RuntimeError("nvcc failed:\n" + failed)
    r = subprocess.run([_nvcc(), *ARCH, "-shared", "-o", LIB, *objects], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("linking failed:\n" + r.stdout + r.stderr)
    build_native(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
