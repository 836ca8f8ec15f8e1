"""Builds libpsgd.so (sm_100a) in-tree with nvcc, and _call.so beside it.  `python -m paper_2509_11254_b200.build`."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", f) for f in ("psgd_api.cu", "psgd_lm.cu", "psgd_layer.cu")]     # compiled side by side
LIB = os.path.join(HERE, "libpsgd.so")
CALL_SRC = os.path.join(HERE, "csrc", "psgd_call.cpp")
CALL = os.path.join(HERE, "_call.so")             # the short way from torch's tensors to the library for small calls
OBJ_DIR = os.path.join(HERE, "_build")
HEADER = os.path.join(os.path.dirname(HERE), "include", "psgd.h")


def nvcc_path():
    for p in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if p and (os.path.isabs(p) and os.path.exists(p) or not os.path.isabs(p)):
            return p
    return "nvcc"


def _torch_dir():
    """Where torch is installed, without importing it."""
    return os.path.dirname(importlib.util.find_spec("torch").origin)


def needs_build():
    if not os.path.exists(LIB) or not os.path.exists(CALL):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALL))
    deps = [HEADER] + [os.path.join(HERE, "csrc", f) for f in os.listdir(os.path.join(HERE, "csrc"))]
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def build_library(force=False, verbose=False):
    if not force and not needs_build():
        return LIB
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xptxas", "-v" if verbose else "-O3",
             "-Xcompiler", "-fPIC"]
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs = [os.path.join(OBJ_DIR, os.path.basename(s)[:-3] + ".o") for s in SRCS]
    jobs = [subprocess.Popen([nvcc_path(), *flags, "-c", "-o", o, s], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            for s, o in zip(SRCS, objs)]
    call_obj = os.path.join(OBJ_DIR, "psgd_call.o")
    torch_dir, cxx = _torch_dir(), os.environ.get("CXX", "g++")
    include = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), sysconfig.get_path("include"),
               os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "include")]
    jobs.append(subprocess.Popen([cxx, "-O2", "-std=c++17", "-fPIC", *(f for p in include for f in ("-isystem", p)), "-c", "-o", call_obj, CALL_SRC], stdout=subprocess.PIPE,
                                 stderr=subprocess.STDOUT, text=True))
    said = [j.communicate()[0] for j in jobs]
    if any(j.returncode != 0 for j in jobs):
        raise RuntimeError("the compiler failed:\n" + "".join(said))
    res = subprocess.run([nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB, *objs], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    # beside the library, which it finds by its own place; torch's are there once torch is imported
    res = subprocess.run([cxx, "-shared", "-o", CALL, call_obj, "-L" + HERE, "-l:libpsgd.so", "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu",
                          "-lc10", "-lc10_cuda"], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("linking _call.so failed:\n" + res.stdout + res.stderr)
    if verbose:
        print("".join(said))
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
