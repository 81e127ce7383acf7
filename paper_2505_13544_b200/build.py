"""Builds libmtla.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(os.path.dirname(PKG_DIR), "include")
LIB_PATH = os.path.join(PKG_DIR, "libmtla.so")
SOURCES = ["mtla_api.cu", "ops_api.cu", "tree_api.cu", "qweight_api.cu"]
OBJ_DIR = os.path.join(PKG_DIR, "_build")


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths += [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    return max(os.path.getmtime(p) for p in paths)


def _nvcc() -> list[str]:
    return [os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a"]


def compile_command(source: str, verbose: bool = False) -> list[str]:
    cmd = _nvcc() + ["-lineinfo", "-O3", "-std=c++17", "-c", "-Xcompiler", "-fPIC", "-I", INCLUDE,
                     "-I", CSRC, "-o", os.path.join(OBJ_DIR, source + ".o")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    return cmd + [os.path.join(CSRC, source)]


def link_command() -> list[str]:
    return _nvcc() + ["-shared", "-o", LIB_PATH] + [os.path.join(OBJ_DIR, s + ".o") for s in SOURCES]


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library if it is missing or older than its sources; returns its path.  The
    translation units are compiled side by side."""
    if (not force and os.path.exists(LIB_PATH)
            and os.path.getmtime(LIB_PATH) >= _newest_source_mtime()):
        return LIB_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)
    procs = [subprocess.Popen(compile_command(s, verbose), stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
             for s in SOURCES]
    outputs = [p.communicate() for p in procs]
    for proc, (out, err) in zip(procs, outputs):
        if verbose:
            sys.stderr.write(err)
        if proc.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + out + err)
    link = subprocess.run(link_command(), capture_output=True, text=True)
    if link.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + link.stdout + link.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
