"""Builds the CUDA library (sm_100a) into paper_2503_01840_b200/libspec_b200.so with nvcc.

    python -m paper_2503_01840_b200.build [--force] [--verbose]

nvcc cross-compiles without a GPU; the resulting .so is loaded by `binding` through ctypes.  g++ compiles _marshal.*.so, the part of the
binding that takes torch tensors apart in C++ for the operators beside the step; each is built for itself where `binding` finds it missing or stale.
"""
import concurrent.futures
import importlib.metadata
import os
import re
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libspec_b200.so")
SOURCES = ["api.cu", "elementwise.cu", "gemm_ref.cu", "tma_maps.cu", "gemm_fused.cu", "gemm_wide.cu", "attn_ref.cu", "attn_fast.cu",
           "attn_causal.cu", "tree.cu", "kv_cache.cu", "attn_decode.cu", "attn_decode_fma.cu", "attn_decode_mma.cu",
           "embedding.cu", "rms_norm.cu", "distill.cu"]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
         "--expt-relaxed-constexpr"]


def _stale(target, ends):
    """Whether target is missing or older than the sources that end like this"""
    if not os.path.exists(target):
        return True
    newest = max(os.path.getmtime(os.path.join(root, f)) for root in (CSRC, os.path.join(os.path.dirname(HERE), "include"))
                 for f in os.listdir(root) if f.endswith(ends))
    return os.path.getmtime(target) < newest


def build_library(force: bool = False, verbose: bool = False) -> str:
    """libspec_b200.so, which SpecDecoder and the C ABI need: nvcc alone makes it."""
    if not force and not _stale(LIB, (".cu", ".cuh", ".h")):
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []

    def cc(src):
        obj = os.path.join(OBJ, src.replace(".cu", ".o"))
        r = subprocess.run([NVCC, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj], capture_output=True, text=True)
        return src, obj, r

    objs = []
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        for src, obj, r in ex.map(cc, SOURCES):
            if verbose or r.returncode:
                sys.stderr.write(f"--- {src}\n{r.stdout}{r.stderr}\n")
            if r.returncode:
                raise RuntimeError(f"nvcc failed on {src}")
            objs.append(obj)
    tmp = LIB + ".%d.tmp" % os.getpid()
    subprocess.run([NVCC, "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a"], check=True)
    os.replace(tmp, LIB)
    return LIB


def marshal_path() -> str:
    """The module's file: made for one Python and one torch, whose names it carries, so that another one's is never loaded."""
    torch_version = re.sub(r"[^A-Za-z0-9.]", "_", importlib.metadata.version("torch"))
    return os.path.join(HERE, f"_marshal.torch-{torch_version}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_marshal(force: bool = False) -> str:
    """The module that the operators beside the step need: with Python's and torch's headers and g++."""
    path = marshal_path()
    if not force and not _stale(path, ("marshal.cpp", ".h")):
        return path
    import torch
    at = os.path.dirname(torch.__file__)
    tmp = path + ".%d.tmp" % os.getpid()
    cuda = os.path.dirname(os.path.dirname(NVCC))
    r = subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
                        *["-I" + d for d in (at + "/include", at + "/include/torch/csrc/api/include", cuda + "/include", sysconfig.get_paths()["include"])],
                        os.path.join(CSRC, "marshal.cpp"), "-o", tmp, "-L" + at + "/lib", "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda",
                        "-Wl,-rpath," + at + "/lib"], capture_output=True, text=True)
    if r.returncode:
        sys.stderr.write(f"--- marshal.cpp\n{r.stdout}{r.stderr}\n")
        raise RuntimeError("the compiler failed on marshal.cpp")
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    """Both; the library's path."""
    with concurrent.futures.ThreadPoolExecutor(max_workers=1) as ex:
        tail = ex.submit(build_marshal, force)
        build_library(force, verbose)
        tail.result()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
