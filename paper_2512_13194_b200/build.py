"""Builds the CUDA library in-tree with nvcc for sm_100a (no GPU needed to compile)."""
from __future__ import annotations

import glob
import hashlib
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libears.so")
UNITS = ("ears_api.cu", "ears_rows_api.cu", "ears_kv_api.cu")      # translation units, compiled side by side
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h"))
                  + [os.path.join(os.path.dirname(HERE), "include", "ears.h")])


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(s) > t for s in sources())


TRACE_LIB = os.path.join(HERE, "libears_trace.so")


def build(force: bool = False, verbose: bool = False, trace: bool = False) -> str:
    """trace=True builds the timeline variant (-DEARS_TRACE: the kernels record the ends of their
    phases, see bench.py --timeline) next to the ordinary library, which it never replaces."""
    out = TRACE_LIB if trace else LIB
    if not force and os.path.exists(out) and all(os.path.getmtime(s) <= os.path.getmtime(out) for s in sources()):
        return out
    flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + (["-DEARS_TRACE"] if trace else [])
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, u[:-3] + ".o") for u in UNITS]
        jobs = [subprocess.Popen([_nvcc()] + flags + ["-c", "-o", o, os.path.join(CSRC, u)]) for u, o in zip(UNITS, objects)]
        codes = [j.wait() for j in jobs]
        for u, code in zip(UNITS, codes):
            if code:
                raise subprocess.CalledProcessError(code, f"nvcc -c {u}")
        linked = f"{out}.{os.getpid()}"      # put in place whole: another process may be loading the library
        subprocess.run([_nvcc()] + NVCC_FLAGS + ["-shared", "-o", linked] + objects, check=True)
        os.replace(linked, out)
    return out


TORCH_LIB = os.path.join(HERE, "ears_torch.so")


def torch_stamp() -> str:
    """What csrc/ears_torch.cpp is compiled from and for, as the module carries it: its source, the C header, torch and Python."""
    import torch
    h = hashlib.sha256(f"{torch.__version__} {sys.version}".encode())
    for path in (os.path.join(CSRC, "ears_torch.cpp"), os.path.join(os.path.dirname(HERE), "include", "ears.h")):
        with open(path, "rb") as f:
            h.update(f.read())
    return "ears_torch:" + h.hexdigest()


def torch_is_stale() -> bool:
    if not os.path.exists(TORCH_LIB):
        return True
    if not os.path.exists(os.path.join(CSRC, "ears_torch.cpp")):
        return False               # a package without its sources
    with open(TORCH_LIB, "rb") as f:
        return torch_stamp().encode() not in f.read()


def build_torch(force: bool = False) -> str:
    """The Python entry of the row operators (csrc/ears_torch.cpp): host code only, against torch's C++ headers."""
    import sysconfig

    import torch
    src = os.path.join(CSRC, "ears_torch.cpp")
    if not force and not torch_is_stale():
        return TORCH_LIB
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    linked = f"{TORCH_LIB}.{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DEARS_TORCH_STAMP="{torch_stamp()}"', f"-I{root}/include",
           f"-I{root}/include/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}/include", "-o", linked, src,
           f"-L{root}/lib", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python", f"-Wl,-rpath,{root}/lib"]
    subprocess.run(cmd, check=True)
    os.replace(linked, TORCH_LIB)
    return TORCH_LIB


if __name__ == "__main__":
    print(build_torch(force="--force" in sys.argv))
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, trace="--trace" in sys.argv))
