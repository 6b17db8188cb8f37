"""Builds in-tree, next to this file: the CUDA library (sm_100a only) with nvcc, libceca_b200.so, and the Python module of
the language-model operators with g++ and torch's headers, _lm_module.*.so.  The library needs neither of those, and is
built without the module where only the ctypes binding is used."""
import glob
import importlib.metadata
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libceca_b200.so")
MODULE_NAME = "_lm_module"
MODULE_SOURCE = os.path.join(CSRC, "lm_module.cc")
HEADER = os.path.join(ROOT, "include", "ceca.h")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xptxas=-v", "-shared", "-Xcompiler", "-fPIC", "--threads", "8"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def module_path():
    """The module for this Python and this torch, whose binary interfaces it uses: another version of either gets its own."""
    return os.path.join(HERE, "%s.%s.torch-%s.so" % (MODULE_NAME, sys.implementation.cache_tag, importlib.metadata.version("torch")))


def _older(path, deps):
    return not os.path.exists(path) or any(os.path.getmtime(f) > os.path.getmtime(path) for f in deps)


def is_stale():
    return _older(LIB, sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + [HEADER])


def module_is_stale():
    return _older(module_path(), [MODULE_SOURCE, HEADER])


def module_command(out):
    """The g++ command of the Python module: torch's own headers and libraries, the CUDA library by its place."""
    import sysconfig

    import torch
    root = os.path.join(os.path.dirname(torch.__file__))
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"),
                os.path.join(ROOT, "include")]
    libs = os.path.join(root, "lib")
    return (["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-DTORCH_EXTENSION_NAME=" + MODULE_NAME, "-DTORCH_API_INCLUDE_EXTENSION_H",
             "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)] + ["-I" + i for i in includes] +
            [MODULE_SOURCE, "-o", out, "-L" + libs, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10_cuda", "-lc10",
             "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN:" + libs])


def _run(what, cmd, verbose):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout)
        print(res.stderr)
    if res.returncode != 0:
        raise RuntimeError(what + " failed")


def build_library(force=False, verbose=False):
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    _run("nvcc", [nvcc] + NVCC_FLAGS + ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", tmp] + sources(), verbose)
    os.replace(tmp, LIB)
    return LIB


def build_module(force=False, verbose=False):
    path = module_path()
    if not force and not module_is_stale():
        return path
    tmp = path + ".tmp.%d" % os.getpid()
    _run("g++", module_command(tmp), verbose)
    os.replace(tmp, path)
    return path


def build(force=False, verbose=False):
    build_library(force, verbose)
    build_module(force, verbose)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
