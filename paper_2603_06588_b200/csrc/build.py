"""Compile the CUDA library for sm_100a into ``libhook_attn.so`` next to the Python binding, and the binding's compiled
part into ``_marshal.so`` beside it.

Every ``.cu`` file is compiled to an object of its own (in parallel, only when it or a header it
includes has changed) under ``_build/`` and the objects are linked into the shared library.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(HERE)
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libhook_attn.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
MARSHAL_SRC = os.path.join(HERE, "marshal.cpp")
OBJ_DIR = os.path.join(HERE, "_build")

FLAGS = ["-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a",
         "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", HERE]


def sources():
    return sorted(glob.glob(os.path.join(HERE, "*.cu")))


def headers():
    return glob.glob(os.path.join(HERE, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _newer(deps, target) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _marshal_stale() -> bool:
    """Older than its sources, or made for another torch or Python than these, which it says when it is imported."""
    if _newer([MARSHAL_SRC] + headers(), MARSHAL):
        return True
    try:
        from .. import _marshal  # noqa: F401
    except ImportError:
        return True
    return False


def needs_build() -> bool:
    return _newer(sources() + headers(), LIB) or _marshal_stale()


def _build_marshal(verbose: bool) -> None:
    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")), "..", "include")
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-Wall", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"),
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", f'-DHOOK_TORCH_VERSION="{torch.__version__}"']
    for path in (os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], cuda):
        cmd += ["-isystem", path]
    cmd += [MARSHAL_SRC, "-o", MARSHAL, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise subprocess.CalledProcessError(res.returncode, res.args)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    hdrs = headers()
    jobs = []
    for src in sources():
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        if force or _newer([src] + hdrs, obj):
            cmd = [nvcc] + FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
            jobs.append(cmd)
    with ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 1))) as pool:
        for res in pool.map(lambda c: subprocess.run(c, capture_output=True, text=True), jobs):
            if verbose or res.returncode != 0:
                sys.stderr.write(res.stdout + res.stderr)
            if res.returncode != 0:
                raise subprocess.CalledProcessError(res.returncode, res.args)
    objs = [os.path.join(OBJ_DIR, os.path.basename(s)[:-3] + ".o") for s in sources()]
    subprocess.run([nvcc, "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB] + objs,
                   check=True)
    if force or _marshal_stale():        # last: the attention's calls do without it
        _build_marshal(verbose)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
