"""Builds libgpd.so (the C-ABI CUDA library, nvcc for sm_100a) and _lm.so (the compiled part of the Python
binding of its low-precision operators, host compiler and torch headers) in-tree.

Usage:  python paper_1811_10751_b200/build.py [--force] [--verbose] [--ptxas]
(run as a script so that the package, which needs the built library, is not imported)
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(PKG_DIR, "_build")
LIB_PATH = os.path.join(PKG_DIR, "libgpd.so")
BINDING_SRC = os.path.join(CSRC, "lm_binding.cpp")
BINDING_PATH = os.path.join(PKG_DIR, "_lm.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _headers_mtime() -> float:
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    hs += [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE) if f.endswith(".h")]
    return max(os.path.getmtime(h) for h in hs)


def _binding_for() -> str:
    """What _lm.so is compiled against: its binary interface is that of one torch and one Python."""
    from importlib import metadata
    return f"torch {metadata.version('torch')} {sys.implementation.cache_tag}"


def _recorded(path: str) -> str:
    try:
        with open(path) as f:
            return f.read()
    except OSError:
        return ""


def _binding_cmd(out: str):
    """Command that compiles and links _lm.so; torch and CUDA runtime libraries are the ones torch has loaded."""
    import sysconfig
    from torch.utils.cpp_extension import include_paths, library_paths
    inc = [f for d in (INCLUDE, sysconfig.get_paths()["include"], *include_paths(device_type="cuda")) for f in ("-I", d)]
    libs = [f for d in (PKG_DIR, *library_paths(device_type="cuda")) for f in ("-L", d)]
    import torch
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *inc, BINDING_SRC, "-o", out, *libs,
            "-lgpd", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    nvcc = _nvcc()
    hm = _headers_mtime()
    jobs = []
    objs = []
    for src in sources():
        obj = os.path.join(BUILD_DIR, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        stale = force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), hm)
        if stale:
            jobs.append([nvcc, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or r.returncode != 0:
            sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"{os.path.basename(cmd[0])} failed: {' '.join(cmd)}")

    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        list(ex.map(run, jobs))
    if jobs or force or not os.path.exists(LIB_PATH):
        tmp = LIB_PATH + f".tmp{os.getpid()}"          # linked aside, then moved: readers never see half a file
        run([nvcc, "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])
        os.replace(tmp, LIB_PATH)
    newest = max(os.path.getmtime(BINDING_SRC), os.path.getmtime(os.path.join(INCLUDE, "gpd.h")))
    built_for, record = _binding_for(), os.path.join(BUILD_DIR, "_lm.built_for")
    if (force or not os.path.exists(BINDING_PATH) or os.path.getmtime(BINDING_PATH) < newest or _recorded(record) != built_for):
        tmp = BINDING_PATH + f".tmp{os.getpid()}"
        run(_binding_cmd(tmp))
        os.replace(tmp, BINDING_PATH)
        with open(record, "w") as f:
            f.write(built_for)
    return LIB_PATH


if __name__ == "__main__":
    flags = ["-Xptxas", "-v"] if "--ptxas" in sys.argv else []
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv or bool(flags), extra_flags=flags))
