"""Build the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the marshalling of the operators' tensors with g++."""
import importlib.util
import os
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
MARSHAL_SRC, MARSHAL = os.path.join(CSRC, "marshal.cpp"), os.path.join(HERE, "_marshal.so")


def _newer(target, deps):
    """Whether target is there and no dependency has changed since."""
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.exists(d) and os.path.getmtime(d) <= t for d in deps)


def needs_build():
    return not _newer(OUT, DEPS) or not _newer(MARSHAL, [MARSHAL_SRC, HEADER])


def _run(cmd, what, verbose=False):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(what + " failed")
    if verbose:
        sys.stderr.write(res.stderr)


def _marshal():
    """The extension module that hands torch tensors to the library (linked against it, so it follows it)."""
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    tmp = MARSHAL + ".new"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-o", tmp, MARSHAL_SRC, "-I" + os.path.join(torch, "include"),
          "-I" + os.path.join(torch, "include", "torch", "csrc", "api", "include"), "-I" + sysconfig.get_paths()["include"], "-I/usr/local/cuda/include",
          "-L" + HERE, "-l:libloopspec.so", "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10",
          "-lc10_cuda"], "g++")
    os.replace(tmp, MARSHAL)


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


def build(force=False, verbose=False):
    if not force and not needs_build():
        return OUT
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    if force or not _newer(OUT, DEPS):
        with ThreadPoolExecutor(len(SRCS)) as pool:
            objs = list(pool.map(lambda s: _object(s, nvcc, force, verbose), SRCS))
        tmp = OUT + ".new"  # (a library that another process has loaded is replaced, not written into)
        _run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp] + objs, "nvcc")
        os.replace(tmp, OUT)
    if force or not _newer(MARSHAL, [MARSHAL_SRC, HEADER]):
        _marshal()
    return OUT


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv)
    print(OUT)
