"""Build the CUDA library (sm_100a only) in-tree, paper_2410_01805_b200/liblocret.so, and the Python module that calls it
without ctypes, _paged.so."""

from __future__ import annotations

import glob
import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblocret.so")
MODULE = os.path.join(HERE, "_paged.so")
MODULE_SRC = os.path.join(CSRC, "paged_module.cpp")
HEADER = os.path.join(HERE, "..", "include", "locret.h")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def built_for() -> str:
    """The torch and Python that the module is compiled against: part of its documentation string, so that another one is noticed."""
    return f"torch {importlib.metadata.version('torch')}, {sysconfig.get_config_var('SOABI')}"


def module_needs_build() -> bool:
    if not os.path.exists(MODULE) or any(os.path.getmtime(p) > os.path.getmtime(MODULE) for p in (MODULE_SRC, HEADER)):
        return True
    with open(MODULE, "rb") as f:
        return f"({built_for()})".encode() not in f.read()


def module_command():
    """g++ against torch's headers and libraries (found without importing it); the library is looked for beside the module."""
    torch = list(importlib.util.find_spec("torch").submodule_search_locations)[0]
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", *("-I" + p for p in include),
            f'-DBUILT_FOR="{built_for()}"', MODULE_SRC, "-o", MODULE, "-L" + HERE, "-l:liblocret.so", "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch",
            "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN"]


def build(force: bool = False, verbose: bool = False) -> str:
    if force or needs_build():
        build_library(force, verbose)
    if force or module_needs_build():
        try:
            subprocess.check_call(module_command())
        except (OSError, subprocess.CalledProcessError) as e:
            raise RuntimeError("the library is built, the module for the calls on pages is not: it needs g++ and the headers of Python "
                               f"and torch ({e}).  All else of the package works without it.") from e
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    os.makedirs(os.path.join(HERE, "build"), exist_ok=True)
    procs = []
    for src in sources():
        obj = os.path.join(HERE, "build", os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if (not force and os.path.exists(obj)
                and os.path.getmtime(obj) > max(os.path.getmtime(src),
                                                *[os.path.getmtime(p) for p in glob.glob(os.path.join(CSRC, "*.cuh"))],
                                                os.path.getmtime(os.path.join(HERE, "..", "include", "locret.h")))):
            continue
        cmd = [nvcc, *NVCC_FLAGS, *os.environ.get("LOCRET_EXTRA_NVCC", "").split(), "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas"); cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write(f"--- {os.path.basename(src)}\n{out}\n")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.check_call([nvcc, "-shared", "-Wno-deprecated-gpu-targets", "-o", LIB, *objs,
                           "-lcudart_static", "-ldl", "-lrt", "-lpthread"])


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
