"""Builds libblr.so (the C-ABI BD-LRU scan library) in-tree with nvcc for sm_103a.

    python -m paper_2406_12580_gb300.build [--verbose]
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBRARY = os.path.join(PKG, "libblr.so")
SOURCES = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))
DEPENDS = SOURCES + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))] + [
    os.path.join(INCLUDE, "blr.h")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc_path() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def nvcc_flags(verbose: bool = False) -> list:
    cuda_lib = os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "lib64")
    flags = [*ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
             "-Xcompiler", "-fvisibility=hidden", "-cudart", "shared", "-I", INCLUDE, "-I", CSRC,
             "-Xlinker", f"-rpath,{cuda_lib}"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    return flags


def stale() -> bool:
    if not os.path.exists(LIBRARY):
        return True
    t = os.path.getmtime(LIBRARY)
    return any(os.path.getmtime(f) > t for f in DEPENDS)


def build(verbose: bool = False, force: bool = True) -> str:
    """Compile the library (atomically replacing any previous build)."""
    if not force and not stale():
        return LIBRARY
    tmp = tempfile.mkdtemp(dir=PKG)
    try:
        flags = nvcc_flags(verbose)

        def run(args: list) -> str:
            res = subprocess.run([nvcc_path(), *flags, *args], stdout=subprocess.PIPE,
                                 stderr=subprocess.STDOUT, text=True)
            if res.returncode != 0:
                raise RuntimeError("nvcc failed:\n" + res.stdout)
            return res.stdout

        objects = [os.path.join(tmp, os.path.basename(f)[:-3] + ".o") for f in SOURCES]
        with concurrent.futures.ThreadPoolExecutor() as pool:  # one nvcc per source file
            texts = list(pool.map(lambda fo: run(["-c", fo[0], "-o", fo[1]]), zip(SOURCES, objects)))
        linked = os.path.join(tmp, "libblr.so")
        texts.append(run(["-shared", *objects, "-o", linked]))
        if verbose:
            sys.stdout.write("".join(texts))
        os.replace(linked, LIBRARY)
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
    return LIBRARY


if __name__ == "__main__":
    build(verbose="--verbose" in sys.argv)
    print(LIBRARY)
