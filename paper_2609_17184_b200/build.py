"""Build the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the marshalling of the operators' tensors with g++.

The library alone needs neither torch nor g++: the marshalling, which is compiled against torch's and Python's headers, is a file of its own, named after
both, that the first call of an operator looks for."""
import importlib.util
import os
import re
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SRCS = [os.path.join(CSRC, "loopspec.cu"), os.path.join(CSRC, "ops.cu")]  # the decode path; the operators around its linear maps
OUT = os.path.join(HERE, "libloopspec.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "loopspec.h")
DEPS = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))] + [HEADER]
MARSHAL_SRC = os.path.join(CSRC, "marshal.cpp")


def _newer(target, deps):
    """Whether target is there and no dependency has changed since."""
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.exists(d) and os.path.getmtime(d) <= t for d in deps)


def needs_build():
    return not _newer(OUT, DEPS)


def torch_dir():
    """Where torch is installed, found without importing it; None where it is not."""
    spec = None if sys.modules.get("torch", True) is None else importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec else None


def marshal_path(torch):
    """The extension module's file for this Python and the torch in that folder: another one of either has no module yet, instead of one that does not load."""
    version = re.search(r"""^__version__ = ['"]([^'"]*)""", open(os.path.join(torch, "version.py")).read(), re.M).group(1)
    return os.path.join(HERE, f"_marshal.{sys.implementation.cache_tag}.torch-{version}.so")


def marshal_needs_build(torch):
    return not _newer(marshal_path(torch), [MARSHAL_SRC, HEADER])


def _run(cmd, what, verbose=False):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(what + " failed")
    if verbose:
        sys.stderr.write(res.stderr)


def build_marshal(torch, force=False):
    """The extension module that hands torch tensors to the library (linked against it, so it follows it)."""
    path = marshal_path(torch)
    if not force and not marshal_needs_build(torch):
        return path
    tmp = f"{path}.{os.getpid()}"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-o", tmp, MARSHAL_SRC, "-I" + os.path.join(torch, "include"),
          "-I" + os.path.join(torch, "include", "torch", "csrc", "api", "include"), "-I" + sysconfig.get_paths()["include"], "-I/usr/local/cuda/include",
          "-L" + HERE, "-l:libloopspec.so", "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10",
          "-lc10_cuda"], "g++")
    os.replace(tmp, path)
    return path


def _object(src, nvcc, force, verbose):
    """One translation unit, compiled unless its object is up to date with the headers it included the last time."""
    obj = src[:-3] + ".o"
    dep = obj + ".d"
    if not force and os.path.exists(dep):
        names = open(dep).read().replace("\\\n", " ").split(":", 1)[-1].split()
        if names and _newer(obj, names):
            return obj
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC",
           "-MD", "-MF", dep, "-c", "-o", obj, src]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    _run(cmd, "nvcc", verbose)
    return obj


def build_library(force=False, verbose=False):
    if not force and not needs_build():
        return OUT
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    with ThreadPoolExecutor(len(SRCS)) as pool:
        objs = list(pool.map(lambda s: _object(s, nvcc, force, verbose), SRCS))
    tmp = OUT + ".new"  # (a library that another process has loaded is replaced, not written into)
    _run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp] + objs, "nvcc")
    os.replace(tmp, OUT)
    return OUT


def build(force=False, verbose=False):
    """The library and, where torch is installed, the marshalling."""
    build_library(force, verbose)
    if torch_dir():
        build_marshal(torch_dir(), force)
    return OUT


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv)
    print(OUT)
