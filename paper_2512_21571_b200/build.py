"""Builds libnnc.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a.  No GPU is needed to build."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libnnc.so")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    d = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    d.append(os.path.join(os.path.dirname(_HERE), "include", "nnc.h"))
    return d


LIB_CHECKED = os.path.join(_HERE, "libnnc_checked.so")   # the same sources with -DNNC_BOUNDS_CHECK (debugging build)


def _compile(src: str, verbose: bool, checked: bool = False) -> str:
    obj = src[:-3] + (".checked.o" if checked else ".o")
    newest_dep = max(os.path.getmtime(p) for p in _deps() + [src])
    if os.path.exists(obj) and os.path.getmtime(obj) >= newest_dep:
        return obj
    cmd = ["nvcc", *NVCC_FLAGS, *(["-DNNC_BOUNDS_CHECK"] if checked else []), "-c", src, "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(r.stderr)
    return obj


CALLS = os.path.join(_HERE, "_calls.so")   # marshalling of the paged-cache operations for torch tensors (csrc/torch_calls.cpp)


def build_calls(force: bool = False) -> str:
    """Builds the extension module _calls.so with g++ against the headers of the running Python and torch; again when its sources
    change, and when it was built for another Python or torch or with another command (CALLS.stamp says which)."""
    import sys
    import sysconfig
    import torch
    src = os.path.join(CSRC, "torch_calls.cpp")
    root = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    compiler = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                *["-I" + i for i in include]]
    libraries = ["-L" + os.path.join(root, "lib"), "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ltorch_python"]
    stamp = "\n".join([sys.version, torch.__version__, *compiler, *libraries])   # (wherever this tree lies)
    newest = max(os.path.getmtime(p) for p in (src, os.path.join(os.path.dirname(_HERE), "include", "nnc.h")))
    if not force and os.path.exists(CALLS) and os.path.getmtime(CALLS) >= newest and os.path.exists(CALLS + ".stamp"):
        with open(CALLS + ".stamp") as f:
            if f.read() == stamp:
                return CALLS
    r = subprocess.run([*compiler, src, "-o", CALLS + ".new", *libraries], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for {src}:\n{r.stdout}\n{r.stderr}")
    os.replace(CALLS + ".new", CALLS)
    with open(CALLS + ".stamp", "w") as f:
        f.write(stamp)
    return CALLS


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Builds libnnc.so, or with checked=True the bounds-checked debugging build libnnc_checked.so; and _calls.so, which serves both."""
    lib = LIB_CHECKED if checked else LIB
    if force:
        for s in sources():
            o = s[:-3] + (".checked.o" if checked else ".o")
            if os.path.exists(o):
                os.remove(o)
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        calls = ex.submit(build_calls, force)
        objs = list(ex.map(lambda s: _compile(s, verbose, checked), sources()))
        calls.result()
    if force or not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(o) for o in objs):
        cmd = ["nvcc", "-shared", "-o", lib, *objs, "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static"]
        subprocess.check_call(cmd)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
