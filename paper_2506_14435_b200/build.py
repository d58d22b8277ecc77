"""Builds libmote.so (sm_100a) in-tree with nvcc, and _calls.so, the extension module of the binding, with g++ against torch.
Usage: python -m paper_2506_14435_b200.build"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libmote.so")
CALLS = os.path.join(PKG, "_calls.so")

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
# never -use_fast_math: the pinned fp32 sequences need IEEE division and no flush-to-zero
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _newest_header():
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    hs.append(os.path.join(ROOT, "include", "mote.h"))
    return max(os.path.getmtime(h) for h in hs)


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJ, src[:-3] + ".o")
    spath = os.path.join(CSRC, src)
    if os.path.exists(obj) and os.path.getmtime(obj) > max(os.path.getmtime(spath), _newest_header()):
        return obj
    cmd = [NVCC, *FLAGS, "-c", spath, "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or r.returncode:
        sys.stderr.write(r.stdout + r.stderr)
    if r.returncode:
        raise RuntimeError("nvcc failed on " + src)
    return obj


def _compile_calls() -> str:
    """torch_calls.cpp -> an object file for the installed torch (its C++ interface is not stable between versions)."""
    import torch
    src = os.path.join(CSRC, "torch_calls.cpp")
    obj = os.path.join(OBJ, f"torch_calls-{torch.__version__}-{sys.implementation.cache_tag}.o")
    if os.path.exists(obj) and os.path.getmtime(obj) > max(os.path.getmtime(src), _newest_header()):
        return obj
    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I" + os.path.join(ROOT, "include"), "-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", cuda, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("g++ failed on torch_calls.cpp")
    return obj


def _link_calls(obj: str) -> None:
    """The extension module from its object file.  Objects of several torch versions can lie side by side: what the module was linked from is
    noted, since an older object may be another version's."""
    note, source = os.path.join(OBJ, "_calls.linked"), f"{obj} {os.path.getmtime(obj)}"
    if os.path.exists(CALLS) and os.path.exists(note):
        with open(note) as f:
            if f.read() == source:
                return
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-shared", "-o", CALLS, obj, "-L" + PKG, "-l:libmote.so", "-Wl,-rpath,$ORIGIN", "-L" + libs,
           "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link of _calls.so failed")
    with open(note, "w") as f:
        f.write(source)


def build(verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=8) as ex:
        calls = ex.submit(_compile_calls)
        objs = list(ex.map(lambda s: _compile(s, verbose), _sources()))
    if not os.path.exists(LIB) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        cmd = [NVCC, "-shared", "-o", LIB, *objs, "-cudart", "static"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link failed")
    _link_calls(calls.result())
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
