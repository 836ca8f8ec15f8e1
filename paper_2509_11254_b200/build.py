"""Builds libpsgd.so (sm_100a) in-tree with nvcc, and, where torch is installed, _call.so beside it.  `python -m paper_2509_11254_b200.build`."""
from __future__ import annotations

import importlib.util
import os
import re
import subprocess
import sys
import sysconfig
import warnings

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
    """Where torch is installed, without importing it; None where it is not."""
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec is not None else None


def _older(built, sources):
    return not os.path.exists(built) or any(os.path.getmtime(d) > os.path.getmtime(built) for d in sources if os.path.exists(d))


def needs_library():
    return _older(LIB, [HEADER] + [os.path.join(HERE, "csrc", f) for f in os.listdir(os.path.join(HERE, "csrc")) if not f.endswith(".cpp")])


def call_tag():
    """What _call.so is compiled against, torch's version (without importing it) and the interpreter; it holds this text."""
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        version = re.search(r"^__version__ *=.*['\"](.+)['\"]", f.read(), re.M)
    return f"psgd_call for torch {version.group(1) if version else '?'}, {sys.implementation.cache_tag}"


def call_fits():
    """Whether _call.so is there and was compiled against this torch and this interpreter."""
    try:
        with open(CALL, "rb") as f:
            return call_tag().encode() + b"\0" in f.read()
    except OSError:
        return False


def needs_call():
    """Where torch is not installed there is nothing to call the library from."""
    return _torch_dir() is not None and (_older(CALL, [HEADER, CALL_SRC]) or not call_fits())


def needs_build():
    return needs_library() or needs_call()


def _start(command):
    return subprocess.Popen(command, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _start_call():
    torch_dir = _torch_dir()
    include = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), sysconfig.get_path("include"),
               os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "include")]
    return _start([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", f'-DPSGD_CALL_BUILT_FOR="{call_tag()}"', *(f for p in include for f in ("-isystem", p)), "-c", "-o", os.path.join(OBJ_DIR, "psgd_call.o"), CALL_SRC])


def _finish_call(job):
    """Links _call.so from what `job` compiles; what went wrong, or None."""
    said = job.communicate()[0]
    if job.returncode != 0:
        return said
    # beside the library, which it finds by its own place; torch's are there once torch is imported
    job = _start([os.environ.get("CXX", "g++"), "-shared", "-o", CALL, os.path.join(OBJ_DIR, "psgd_call.o"), "-L" + HERE, "-l:libpsgd.so", "-Wl,-rpath,$ORIGIN",
                  "-L" + os.path.join(_torch_dir(), "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    said = job.communicate()[0]
    return said if job.returncode != 0 else None


def build_library(force=False, verbose=False):
    """Builds what is missing or older than its sources.  The library needs nvcc alone; where _call.so, which needs a C++ compiler and the headers of Python and torch too, cannot be
    built, a warning says why."""
    library, call = force or needs_library(), _torch_dir() is not None and (force or needs_call())
    if not library and not call:
        return LIB
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xptxas", "-v" if verbose else "-O3",
             "-Xcompiler", "-fPIC"]
    os.makedirs(OBJ_DIR, exist_ok=True)
    why = job = None
    if call:
        try:
            job = _start_call()
        except OSError as e:                          # (no such compiler)
            why = str(e)
    if library:
        objs = [os.path.join(OBJ_DIR, os.path.basename(s)[:-3] + ".o") for s in SRCS]
        jobs = [_start([nvcc_path(), *flags, "-c", "-o", o, s]) for s, o in zip(SRCS, objs)]
        said = [j.communicate()[0] for j in jobs]
        if any(j.returncode != 0 for j in jobs):
            if job is not None:
                job.communicate()
            raise RuntimeError("nvcc failed:\n" + "".join(said))
        link = _start([nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB, *objs])
        text = link.communicate()[0]
        if link.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + text)
        if verbose:
            print("".join(said))
    if job is not None:
        why = _finish_call(job)
    if why is not None:
        warnings.warn(f"_call.so could not be built: {why}", RuntimeWarning, stacklevel=2)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
