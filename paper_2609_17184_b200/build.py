"""Build the CUDA extension in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SRCS = [os.path.join(CSRC, "loopspec.cu"), os.path.join(CSRC, "ops.cu")]  # the decode path; the operators around its linear maps
OUT = os.path.join(HERE, "libloopspec.so")
DEPS = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))] + [
    os.path.join(os.path.dirname(HERE), "include", "loopspec.h")]


def _newer(target, deps):
    """Whether target is there and no dependency has changed since."""
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.exists(d) and os.path.getmtime(d) <= t for d in deps)


def needs_build():
    return not _newer(OUT, DEPS)


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
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed")
    if verbose:
        sys.stderr.write(res.stderr)
    return obj


def build(force=False, verbose=False):
    if not force and not needs_build():
        return OUT
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    with ThreadPoolExecutor(len(SRCS)) as pool:
        objs = list(pool.map(lambda s: _object(s, nvcc, force, verbose), SRCS))
    tmp = OUT + ".new"  # (a library that another process has loaded is replaced, not written into)
    res = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp] + objs, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed")
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv)
    print(OUT)
