"""Builds libpsgd.so (sm_100a) in-tree with nvcc.  `python -m paper_2509_11254_b200.build`."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", f) for f in ("psgd_api.cu", "psgd_lm.cu")]     # compiled side by side
LIB = os.path.join(HERE, "libpsgd.so")
OBJ_DIR = os.path.join(HERE, "_build")
HEADER = os.path.join(os.path.dirname(HERE), "include", "psgd.h")


def nvcc_path():
    for p in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if p and (os.path.isabs(p) and os.path.exists(p) or not os.path.isabs(p)):
            return p
    return "nvcc"


def needs_build():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
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
    said = [j.communicate()[0] for j in jobs]
    if any(j.returncode != 0 for j in jobs):
        raise RuntimeError("nvcc failed:\n" + "".join(said))
    res = subprocess.run([nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB, *objs], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print("".join(said))
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
