"""Builds libadmmq.so (sm_100a) and _adapt.so, its calls from Python, next to this file:
python -m paper_2605_11222_b200.build"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libadmmq.so")
BIND = os.path.join(HERE, "_adapt.so")
BIND_FOR = os.path.join(OBJ, "_adapt.for")     # the Python and the torch that _adapt.so was built for
SOURCES = ["api.cu", "elem.cu", "gemm_simt.cu", "gemm_tc.cu", "tridiag.cu", "tridiag_blocked.cu", "local_search.cu", "pair_swap.cu",
           "objective_static.cu", "adapt_api.cu", "linear_small.cu", "shrink_tc.cu", "linear_tc.cu", "linear_pair.cu", "adapter_grad.cu", "checkpoint8.cu",
           "qk_rope.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _newer(src_paths, target):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(s) > t for s in src_paths)


def build(force: bool = False, verbose: bool = False) -> str:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    include = os.path.join(os.path.dirname(HERE), "include")
    headers += [os.path.join(include, f) for f in os.listdir(include) if f.endswith(".h")]

    def compile_one(name):
        src = os.path.join(CSRC, name)
        obj = os.path.join(OBJ, name.replace(".cu", ".o"))
        if force or _newer([src] + headers, obj):
            r = subprocess.run([nvcc, *NVCC_FLAGS, "-c", src, "-o", obj], capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {name}:\n{r.stdout}\n{r.stderr}")
            if verbose:
                sys.stderr.write(r.stderr)
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=6) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    if force or _newer(objs, LIB):
        r = subprocess.run([nvcc, "-shared", "-o", LIB, *objs, "-lcudart_static", "-ldl", "-lrt", "-lpthread"],
                           capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    _build_bind(force, [h for h in headers if h.startswith(include)])
    return LIB


def _bind_for() -> str:
    """What _adapt.so depends on besides this repository: it uses internals of torch and of the running Python."""
    import torch
    return f"python {sys.version} torch {torch.__version__} abi {int(torch._C._GLIBCXX_USE_CXX11_ABI)}"


def _bind_is_current(sources) -> bool:
    if _newer(sources, BIND) or not os.path.exists(BIND_FOR):
        return False
    with open(BIND_FOR) as f:
        return f.read() == _bind_for()


def _build_bind(force: bool, headers) -> None:
    """The Python calls of the operators (CPython and torch C++, no device code)."""
    src = os.path.join(CSRC, "adapt_bind.cpp")
    if not force and _bind_is_current([src] + headers):
        return
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    lib = os.path.join(root, "lib")
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.environ.get("CUDA_INCLUDE", "/usr/local/cuda/include"), sysconfig.get_paths()["include"]]
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    r = subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                        f"-D_GLIBCXX_USE_CXX11_ABI={abi}", *[f"-I{i}" for i in inc], src, "-o", BIND, f"-L{lib}", f"-L{HERE}",
                        "-l:libadmmq.so", "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-ltorch", "-lc10_cuda", "-lc10",
                        "-Wl,-rpath,$ORIGIN"], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"building {BIND} failed:\n{r.stdout}\n{r.stderr}")
    with open(BIND_FOR, "w") as f:
        f.write(_bind_for())


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
