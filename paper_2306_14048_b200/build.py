"""Build libh2o_b200.so (the C-ABI library) in-tree with nvcc for sm_100a, and the _pages extension (argument checks of the
paged cache's calls, host code) with the C++ compiler.

``python paper_2306_14048_b200/build.py`` (run as a script, so that the package — which refuses to
import without the library — is not imported first) or ``build()``; the library is rebuilt
only when a source or header is newer than it.  nvcc cross-compiles, so this also
works on a machine without a GPU.
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import re
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "build")
LIB = os.path.join(PKG, "libh2o_b200.so")
LIB_BOUNDS = os.path.join(PKG, "libh2o_b200_bounds.so")  # the same sources with -DH2O_BOUNDS (every index checked)

PAGES_SOURCE = os.path.join(CSRC, "pages_binding.cpp")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(p) > t for p in _deps())


def pages_path() -> str:
    """Where the _pages extension for the running Python and torch lies: it reads tensors by torch's C++ headers, so that one built for
    another of either must not be loaded."""
    import torch

    version = "%s-%s" % (torch.__version__, (torch.version.git_version or "")[:8])
    return os.path.join(PKG, "_pages-torch" + re.sub(r"[^0-9A-Za-z.-]", "_", version) + sysconfig.get_config_var("EXT_SUFFIX"))


def build_pages(force: bool = False) -> str:
    """The _pages extension: host code that reads torch tensors, built where there is none for this Python and torch, or where its
    sources are newer."""
    lib = pages_path()
    newest = max(os.path.getmtime(p) for p in [PAGES_SOURCE] + glob.glob(os.path.join(ROOT, "include", "*.h")))
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= newest:
        return lib
    import torch

    at = os.path.dirname(torch.__file__)
    tmp = lib + ".tmp.%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    for d in (os.path.join(ROOT, "include"), os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
              sysconfig.get_paths()["include"]):
        cmd += ["-I", d]
    cmd += [PAGES_SOURCE, "-o", tmp, "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("%s failed for %s:\n%s\n%s" % (cmd[0], PAGES_SOURCE, res.stdout, res.stderr))
    os.replace(tmp, lib)
    return lib


def build(force: bool = False, verbose: bool = False, bounds: bool = False) -> str:
    """``bounds``: build libh2o_b200_bounds.so instead, the checked variant (-DH2O_BOUNDS)."""
    lib = LIB_BOUNDS if bounds else LIB
    build_pages(force)
    if not force and not needs_build(lib):
        return lib
    nvcc = os.environ.get("NVCC", "nvcc")
    obj_dir = OBJ + ("_bounds" if bounds else "")
    os.makedirs(obj_dir, exist_ok=True)
    extra = (["-Xptxas", "-v"] if verbose else []) + (["-DH2O_BOUNDS"] if bounds else [])

    def compile_one(src):
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc] + NVCC_FLAGS + extra + ["-c", src, "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed for %s:\n%s\n%s" % (src, res.stdout, res.stderr))
        if verbose:
            sys.stderr.write(res.stderr)
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, _sources()))
    tmp = lib + ".tmp.%d" % os.getpid()
    res = subprocess.run([nvcc, "-shared", "-o", tmp] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"],
                         capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (res.stdout, res.stderr))
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, bounds="--bounds" in sys.argv))
