"""Builds libsmoothrot.so in-tree with nvcc for sm_100a.

    python -m paper_2506_05413_b200.build

Objects go to paper_2506_05413_b200/_build/, the library next to this file, and beside it _marshal.so, the
native marshalling of some of the binding's calls.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsmoothrot.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = ("rotate_quant.cu", "calibrate.cu", "w4a4_gemm.cu", "clip_search.cu", "kv_quant.cu", "heads_quant.cu", "decode_fused.cu", "plain_quant.cu",
           "kv_cache.cu", "attn_decode.cu", "attn_prefill.cu")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths.append(os.path.join(ROOT, "include", "smoothrot.h"))
    return max(os.path.getmtime(p) for p in paths)


def is_current() -> bool:
    return all(os.path.exists(p) and os.path.getmtime(p) >= _newest_source_mtime() for p in (LIB, MARSHAL))


def build_marshal() -> str:
    """Compile csrc/marshal.cpp against torch's headers into a Python extension module; returns its path."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    tmp = MARSHAL + f".tmp{os.getpid()}"
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           *("-isystem" + p for p in (*cpp_extension.include_paths(), sysconfig.get_paths()["include"], cuda)),
           os.path.join(CSRC, "marshal.cpp"), "-o", tmp, "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch_cpu",
           "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed on marshal.cpp")
    os.replace(tmp, MARSHAL)
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu file for sm_100a and link the shared library; returns its path.

    The library needs nvcc alone and is linked whatever becomes of the binding's module, which needs torch's headers and a
    C++ compiler: where that fails, the error is raised with the library in place for users of its C interface.
    """
    if not force and is_current():
        return LIB
    nvcc = _nvcc()
    os.makedirs(BUILD, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        cmd = [nvcc, *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
        if res.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as pool:
        marshal = pool.submit(build_marshal)
        objs = list(pool.map(compile_one, SOURCES))
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.check_call([nvcc, "-shared", "-Wno-deprecated-gpu-targets", "-o", tmp, *objs])
        os.replace(tmp, LIB)
        marshal.result()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
