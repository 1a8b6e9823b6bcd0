"""Builds libmhclite.so (nvcc for sm_100a, cross-compiles without a GPU) and the Python extension _marshal.so (the host
compiler against the installed torch) in-tree.

    python -m paper_2601_05732_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import concurrent.futures as cf
import hashlib
import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
OBJ_DIR = os.path.join(PKG_DIR, "_build")
LIB_PATH = os.path.join(PKG_DIR, "libmhclite.so")
MARSHAL_PATH = os.path.join(PKG_DIR, "_marshal.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
    "-rdc=true", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-Xptxas", "-v",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: cannot build libmhclite.so")


def _sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _digest(paths) -> str:
    h = hashlib.sha256()
    for p in sorted(paths):
        h.update(p.encode())
        with open(p, "rb") as f:
            h.update(f.read())
    h.update(" ".join(NVCC_FLAGS).encode())
    return h.hexdigest()


def _all_inputs():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h"))]
    files.append(os.path.join(os.path.dirname(PKG_DIR), "include", "mhclite.h"))
    return files


def build_marshal(force: bool = False) -> str:
    """Compiles csrc/marshal.cpp, the argument marshalling of the calls around the stack; returns the module's path."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    root = os.path.dirname(torch.__file__)
    src, header = os.path.join(CSRC, "marshal.cpp"), os.path.join(os.path.dirname(PKG_DIR), "include", "mhclite.h")
    libs = os.path.join(root, "lib")
    cuda = os.environ.get("CUDA_HOME") or os.path.dirname(os.path.dirname(_nvcc()))
    fresh = os.path.join(OBJ_DIR, f"marshal.{os.getpid()}")           # moved into place whole: several processes may build
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DMHCL_TORCH_VERSION="{torch.__version__}"', f"-I{sysconfig.get_paths()['include']}",
           *[f"-I{p}" for p in cpp_extension.include_paths()], f"-I{os.path.join(cuda, 'include')}", src, "-o", fresh,
           f"-L{libs}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", f"-Wl,-rpath,{libs}"]
    digest = hashlib.sha256("\0".join([*(a for a in cmd if a != fresh), torch.__version__, sys.version, open(src).read(), open(header).read()]).encode()).hexdigest()
    stamp = os.path.join(OBJ_DIR, "marshal.stamp")
    if not force and os.path.exists(MARSHAL_PATH) and os.path.exists(stamp) and open(stamp).read() == digest:
        return MARSHAL_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed on marshal.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(fresh, MARSHAL_PATH)
    with open(stamp, "w") as f:
        f.write(digest)
    return MARSHAL_PATH


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu under csrc/ and links libmhclite.so, after _marshal.so; returns the library's path."""
    build_marshal(force)
    stamp = os.path.join(OBJ_DIR, "stamp")
    digest = _digest(_all_inputs())
    if not force and os.path.exists(LIB_PATH) and os.path.exists(stamp) and open(stamp).read() == digest:
        return LIB_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)
    nvcc = _nvcc()

    def compile_one(src):
        obj = os.path.join(OBJ_DIR, src[:-3] + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        with open(os.path.join(OBJ_DIR, src[:-3] + ".ptxas.log"), "w") as f:
            f.write(r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, _sources()))
    link = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB_PATH, *objs]
    r = subprocess.run(link, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    with open(stamp, "w") as f:
        f.write(digest)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
