"""Builds libet.so (the C-ABI library) in-tree with nvcc for sm_100a, and the binding's helper module _operands with the host compiler.

    python paper_2312_14227_b200/build.py [--force] [--verbose] [--debug-hooks]

Rebuilds only when a source is newer than the library (--force: always).  --debug-hooks compiles the
development switches in (forced tile shapes from the environment); the library built without it
reads nothing from the environment.
"""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libet.so")
SOURCES = ["et_lib.cu", "et_noalloc.cu", "select.cpp"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "py_operands.cpp"] + [os.path.join(ROOT, "include", "et.h")]
    return max(os.path.getmtime(p) for p in paths)


OPERANDS = os.path.join(HERE, "_operands" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
OPERANDS_SOURCE = os.path.join(CSRC, "py_operands.cpp")


def build_operands(force: bool = False, verbose: bool = False):
    """The helper module, where torch and Python's headers are installed; the binding works without it."""
    if not force and os.path.exists(OPERANDS) and os.path.getmtime(OPERANDS) >= os.path.getmtime(OPERANDS_SOURCE):
        return OPERANDS
    spec = importlib.util.find_spec("torch")
    python = sysconfig.get_paths()["include"]
    if spec is None or not spec.submodule_search_locations or not os.path.exists(os.path.join(python, "Python.h")):
        return None
    torch = list(spec.submodule_search_locations)[0]
    cmd = [os.environ.get("CXX", "g++"), "-shared", "-fPIC", "-std=c++17", "-O2", "-o", OPERANDS, OPERANDS_SOURCE, "-I", python,
           "-I", os.path.join(torch, "include"), "-I", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
           "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    try:
        res = subprocess.run(cmd, capture_output=True, text=True)
        failed, said = res.returncode != 0, res.stdout + res.stderr
    except OSError as e:
        failed, said = True, str(e)
    if failed:
        print("_operands was not built, the binding checks lists of tensors in Python:\n" + said, file=sys.stderr)
        return None
    if verbose:
        print(said)
    return OPERANDS


def build(force: bool = False, verbose: bool = False, debug_hooks: bool = False) -> str:
    build_operands(force, verbose)
    return build_library(force, verbose, debug_hooks)


def build_library(force: bool = False, verbose: bool = False, debug_hooks: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [
        nvcc, "-shared", "-o", LIB, "-std=c++17", "-O3", "-lineinfo",
        "-gencode", "arch=compute_100a,code=sm_100a",
        "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=default",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
        "-cudart", "static", "-Xcompiler", "-pthread",
    ]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    if debug_hooks:
        cmd += ["-DET_DEBUG_HOOKS"]
    cmd += [os.path.join(CSRC, f) for f in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stdout + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv or "--debug-hooks" in sys.argv, verbose="--verbose" in sys.argv,
                debug_hooks="--debug-hooks" in sys.argv))
