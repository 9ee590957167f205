"""Builds libdetox.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the Python module _worker that
calls it (g++, against the installed torch)."""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdetox.so")
MODULE_SRC = os.path.join(PKG, "csrc_py", "worker_module.cpp")
MODULE = os.path.join(PKG, "_worker.so")
MODULE_STAMP = os.path.join(OBJ, "worker_module.txt")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps_mtime():
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    hdrs.append(os.path.join(ROOT, "include", "detox.h"))
    return max(os.path.getmtime(h) for h in hdrs)


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJ, src[:-3] + ".o")
    path = os.path.join(CSRC, src)
    if os.path.exists(obj) and os.path.getmtime(obj) >= max(os.path.getmtime(path), _deps_mtime()):
        return obj
    cmd = ["nvcc", *NVCC_FLAGS, "-c", path, "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{res.stdout}\n{res.stderr}")
    if verbose:
        sys.stderr.write(res.stderr)
    return obj


def _module_command():
    """How the Python module is compiled here, or why it cannot be."""
    import sysconfig

    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    if shutil.which("g++") is None:
        return None, "no g++"
    if not os.path.isdir(os.path.join(inc, "torch")):
        return None, f"no torch headers in {inc}"
    return ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-I", os.path.join(ROOT, "include"), "-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"),
            "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"], MODULE_SRC, "-o", MODULE,
            "-L", PKG, "-l:libdetox.so", "-L", lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda",
            "-Wl,-rpath,$ORIGIN"], None


def _module_stamp() -> str:
    """What the module's binary form depends on beside its source."""
    import torch
    return f"python {sys.version_info[0]}.{sys.version_info[1]}, torch {torch.__version__}\n"


def _build_module(force: bool):
    """The Python module of the worker-side operators; it finds libdetox.so beside itself.  Where it cannot be compiled, the
    aggregation goes without it: a warning here, and an error when one of those operators is called."""
    newest = max(os.path.getmtime(p) for p in (MODULE_SRC, os.path.join(ROOT, "include", "detox.h")))
    stamp = _module_stamp()
    if not force and os.path.exists(MODULE) and os.path.getmtime(MODULE) >= newest:
        if os.path.exists(MODULE_STAMP) and open(MODULE_STAMP).read() == stamp:
            return
    cmd, why = _module_command()
    if cmd is None:
        warnings.warn(f"the worker-side operators are not built: {why}")
        return
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"g++ failed on {MODULE_SRC}:\n{res.stdout}\n{res.stderr}")
    with open(MODULE_STAMP, "w") as f:
        f.write(stamp)


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    if force:
        for f in os.listdir(OBJ):
            if f.endswith(".o"):
                os.remove(os.path.join(OBJ, f))
    srcs = _sources()
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    if force or not os.path.exists(LIB) or os.path.getmtime(LIB) < max(os.path.getmtime(o) for o in objs):
        cmd = ["nvcc", "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB, *objs, "-cudart", "static"]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
    _build_module(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
