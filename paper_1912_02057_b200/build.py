"""Builds librtn_b200.so in-tree with nvcc for sm_100a, and _rtn_torch.so, the torch side of the layer operators, with g++.

Usage: python -m paper_1912_02057_b200.build [--force] [--verbose] [--timeline]

--timeline builds a second library, librtn_b200_timeline.so, with the in-kernel clock stamps of
csrc/rtn_timeline.cuh compiled in (for paper_1912_02057_b200.timeline; the product library never has them).
"""
import glob
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "librtn_b200.so")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _newer(target, deps):
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(d) <= t for d in deps)


LIB_TIMELINE = os.path.join(HERE, "librtn_b200_timeline.so")


def build(force=False, verbose=False, timeline=False):
    if timeline:
        return _build(os.path.join(HERE, "_build_timeline"), LIB_TIMELINE, ["-DRTN_TIMELINE"], force, verbose)
    lib = _build(OBJ, LIB, [], force, verbose)
    _build_torch(force, verbose)
    return lib


LIB_TORCH = os.path.join(HERE, "_rtn_torch.so")


def _build_torch(force, verbose):
    src = os.path.join(CSRC, "rtn_torch.cpp")
    if not force and _newer(LIB_TORCH, [src, os.path.join(ROOT, "include", "rtn.h")]):
        return
    import sysconfig
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    libs = library_paths()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"),
           *(x for i in include_paths() for x in ("-isystem", i)), src, "-o", LIB_TORCH,
           *(x for l in libs for x in ("-L" + l, "-Wl,-rpath," + l)), "-lc10", "-ltorch", "-ltorch_cpu", "-ltorch_python", "-lc10_cuda", "-ltorch_cuda"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or r.returncode != 0:
        sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on rtn_torch.cpp")


def _build(OBJ, LIB, extra, force, verbose):
    os.makedirs(OBJ, exist_ok=True)
    headers = glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    objs, jobs = [], []
    for src in sources:
        obj = os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or not _newer(obj, [src] + headers):
            cmd = ["nvcc", *NVCC_FLAGS, *extra, "-c", src, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            jobs.append(cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    with ThreadPoolExecutor(max_workers=8) as ex:
        for cmd, r in ex.map(run, jobs):
            if verbose or r.returncode != 0:
                sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {cmd[-3]}")
    if jobs or force or not _newer(LIB, objs):
        cmd = ["nvcc", "-shared", "-o", LIB, *objs, "-gencode", "arch=compute_100a,code=sm_100a",
               "-cudart", "static"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link failed")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv, timeline="--timeline" in sys.argv))
