"""Builds ``libmaps.so`` (the C-ABI library) in-tree for sm_103a.

Each ``csrc/*.cu`` is compiled in parallel with nvcc, then linked into one
shared library next to this file.  A source or header newer than the
library triggers a rebuild.  ``csrc/marshal.cpp``, the binding's native
argument marshalling, becomes an extension module of this Python beside it,
built again for another PyTorch; where PyTorch's or Python's headers do not
compile, the binding does that work in Python, and the next build tries again.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import importlib.util
import os
import re
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libmaps.so")
MARSHAL = os.path.join(PKG, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))  # no other Python's

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC",
                     "-Xcompiler", "-O2", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _newer(made: str, inputs: list[str]) -> bool:
    if not os.path.exists(made):
        return False
    t = os.path.getmtime(made)
    return all(os.path.getmtime(f) <= t for f in inputs)


def _headers() -> list[str]:
    return glob.glob(os.path.join(INCLUDE, "*.h")) + [os.path.abspath(__file__)]


def library_up_to_date() -> bool:
    return _newer(LIB, sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + _headers())


def marshal_up_to_date() -> bool:
    try:
        with open(_marshal_key()) as f:
            return f.read() == torch_version() and _newer(MARSHAL, glob.glob(os.path.join(CSRC, "*.cpp")) + _headers())
    except (OSError, AttributeError):
        return False


def up_to_date() -> bool:
    return library_up_to_date() and marshal_up_to_date()


def _torch_root() -> str:
    return os.path.dirname(importlib.util.find_spec("torch").origin)


def torch_version() -> str:
    with open(os.path.join(_torch_root(), "version.py")) as f:
        return re.search(r"__version__ = ['\"]([^'\"]+)", f.read()).group(1)


def _marshal_key() -> str:
    """The file that says which PyTorch the module was built for."""
    return os.path.join(BUILD, os.path.basename(MARSHAL) + ".torch")


def build_marshal() -> None:
    tmp = MARSHAL + f".{os.getpid()}.tmp"
    old = os.path.join(PKG, "_marshal.so")  # of no Python in particular, so any would load it
    if os.path.exists(old) and old != MARSHAL:
        os.remove(old)
    try:
        torch, version = _torch_root(), torch_version()
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f'-DMAPS_TORCH_VERSION="{version}"', "-I", INCLUDE,
               "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(torch, "include"),
               os.path.join(CSRC, "marshal.cpp"), "-o", tmp, "-L", os.path.join(torch, "lib"), "-ltorch_python", "-lc10"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode == 0:
            os.replace(tmp, MARSHAL)
            with open(_marshal_key(), "w") as f:
                f.write(version)
            return
        why = r.stderr[:2000]
    except (OSError, AttributeError) as e:
        why = str(e)
    if os.path.exists(MARSHAL):  # of other sources
        os.remove(MARSHAL)
    print(f"arguments are marshalled in Python: {why}", file=sys.stderr)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    if not force and library_up_to_date():
        build_marshal()
        return LIB
    nvcc = _nvcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr)
        return obj

    srcs = sources()
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs) + 1, os.cpu_count() or 4)) as ex:
        marshal = None if not force and marshal_up_to_date() else ex.submit(build_marshal)
        objs = list(ex.map(compile_one, srcs))
        if marshal is not None:
            marshal.result()
    tmp = LIB + f".{os.getpid()}.tmp"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
