"""Builds libblr.so (the C-ABI BD-LRU scan library) in-tree with nvcc for sm_103a, and
_torch_ext.so (torch tensors to its arguments, autograd) with the C++ compiler.

    python -m paper_2406_12580_gb300.build [--verbose]
"""
from __future__ import annotations

import concurrent.futures
import os
import re
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
EXTENSION = os.path.join(PKG, "_torch_ext.so")
EXTENSION_SOURCE = os.path.join(CSRC, "blr_torch.cpp")
DEPENDS = SOURCES + [EXTENSION_SOURCE] + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))] + [
    os.path.join(INCLUDE, "blr.h")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc_path() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def compiler_path() -> str:
    path = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if path:
        return path
    raise RuntimeError("no C++ compiler found")


def nvcc_flags(verbose: bool = False) -> list:
    cuda_lib = os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "lib64")
    flags = [*ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
             "-Xcompiler", "-fvisibility=hidden", "-cudart", "shared", "-I", INCLUDE, "-I", CSRC,
             "-Xlinker", f"-rpath,{cuda_lib}"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    return flags


def extension_command(compiler: str, library_dir: str, out: str) -> list:
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    lib = os.path.join(root, "lib")
    include = [INCLUDE, os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "include")]
    return [compiler, "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[f"-I{p}" for p in include],
            EXTENSION_SOURCE, "-o", out, f"-L{lib}", f"-L{library_dir}", "-ltorch_python", "-ltorch_cpu", "-ltorch",
            "-lc10", "-lc10_cuda", "-lblr", f"-Wl,-rpath,{lib}:$ORIGIN"]


def stale() -> bool:
    if not os.path.exists(LIBRARY) or not os.path.exists(EXTENSION):
        return True
    t = min(os.path.getmtime(LIBRARY), os.path.getmtime(EXTENSION))
    return any(os.path.getmtime(f) > t for f in DEPENDS)


def build(verbose: bool = False, force: bool = True) -> str:
    """Compile the library (atomically replacing any previous build)."""
    if not force and not stale():
        return LIBRARY
    tmp = tempfile.mkdtemp(dir=PKG)
    try:
        flags = nvcc_flags(verbose)

        def run(command: list) -> str:
            res = subprocess.run(command, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            if res.returncode != 0:
                raise RuntimeError(f"{os.path.basename(command[0])} failed:\n{res.stdout}")
            return res.stdout

        def extension() -> str:  # against a stand-in for the library, which is still being built
            stub = os.path.join(tmp, "stub")
            os.mkdir(stub)
            declared = re.findall(r"^BLR_API\s+[\w\s\*]*?\b(blr_\w+)\s*\(", open(os.path.join(INCLUDE, "blr.h")).read(), re.M)
            with open(os.path.join(stub, "stub.c"), "w") as f:
                f.write("".join(f"void {name}(void) {{}}\n" for name in declared))
            run([compiler_path(), "-xc", "-shared", "-fPIC", "-Wl,-soname,libblr.so", os.path.join(stub, "stub.c"), "-o",
                 os.path.join(stub, "libblr.so")])
            return run(extension_command(compiler_path(), stub, os.path.join(tmp, "_torch_ext.so")))

        objects = [os.path.join(tmp, os.path.basename(f)[:-3] + ".o") for f in SOURCES]
        with concurrent.futures.ThreadPoolExecutor() as pool:  # a compiler for each source file
            other = pool.submit(extension)
            texts = list(pool.map(lambda fo: run([nvcc_path(), *flags, "-c", fo[0], "-o", fo[1]]), zip(SOURCES, objects)))
            texts.append(other.result())
        linked = os.path.join(tmp, "libblr.so")
        texts.append(run([nvcc_path(), *flags, "-shared", "-Xlinker", "-soname,libblr.so", *objects, "-o", linked]))
        if verbose:
            sys.stdout.write("".join(texts))
        os.replace(linked, LIBRARY)
        os.replace(os.path.join(tmp, "_torch_ext.so"), EXTENSION)
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
    return LIBRARY


if __name__ == "__main__":
    build(verbose="--verbose" in sys.argv)
    print(LIBRARY)
