"""Builds the CUDA library in-tree: nvcc for sm_100a -> paper_2507_07149_b200/libdaf.so."""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libdaf.so")
HEADERS = [os.path.join(CSRC, h) for h in ("common.cuh", "compress_shared.cuh", "compress_stream.cuh", "compress_general.cuh", "compress_twopass.cuh", "compress_twowidth.cuh", "attention.cuh", "attention_tc.cuh", "attention_tc_grad.cuh", "tensor_core.cuh", "pairs.cuh", "launch_cache.hpp")] + [
    os.path.join(os.path.dirname(HERE), "include", "daf.h")]

CU_SOURCES = ["api.cu", "compress.cu", "compress_stream_f32.cu", "compress_stream_f16.cu", "compress_stream_bf16.cu", "compress_twowidth_f32.cu", "compress_twowidth_f16.cu", "compress_twowidth_bf16.cu", "compress_twopass_f32.cu", "compress_twopass_f16.cu", "compress_twopass_bf16.cu", "compress_general_f32.cu", "compress_general_f16.cu",
              "compress_general_bf16.cu", "decompress.cu", "group_offsets.cu", "tensorwise.cu",
              "attention.cu", "attention_rows.cu", "attention_tc_f32.cu", "attention_tc_f16.cu", "attention_tc_bf16.cu", "residual_norm.cu", "clip_norm.cu", "embedding.cu", "rotary_norm.cu", "orthogonalize.cu"]
CXX_SOURCES = ["pool.cpp", "store.cpp"]

# The Python module that marshals torch tensors for the transformer operators (host code only).
MARSHAL = os.path.join(HERE, "_marshal.so")
MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")
MARSHAL_MADE = os.path.join(OBJ, "marshal.made")                 # which torch and Python it was built for

# No fast-math, no flush-to-zero, no fused contraction beyond what the sources write out:
# results must match IEEE binary32 arithmetic bit for bit.
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "--fmad=false", "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


# Extra compiler flags for development builds (e.g. -DDAF_STAMPS), read when the library is built.
NVCC_FLAGS += os.environ.get("DAF_NVCC_EXTRA", "").split()


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return exe


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    nvcc = _nvcc()
    jobs = []
    for src in CU_SOURCES + CXX_SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(OBJ, src + ".o")
        if force or _stale(obj, [path] + HEADERS):
            jobs.append((src, [nvcc, *NVCC_FLAGS, "-c", path, "-o", obj]))

    def run(job):
        name, cmd = job
        r = subprocess.run(cmd, capture_output=True, text=True)
        with open(os.path.join(OBJ, name + ".log"), "w") as f:
            f.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {name}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            print(r.stdout + r.stderr)

    with ThreadPoolExecutor(max(1, min(len(jobs), os.cpu_count() or 1))) as ex:
        list(ex.map(run, jobs))
    objs = [os.path.join(OBJ, s + ".o") for s in CU_SOURCES + CXX_SOURCES]
    if force or jobs or _stale(LIB, objs):
        subprocess.check_call([nvcc, "-shared", "-o", LIB, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])
    build_marshal(force)
    return LIB


def build_marshal(force: bool = False) -> str:
    """Compiles csrc/marshal.cpp against torch and libdaf.so (found beside it when the module is loaded).  Without torch there is
    nothing to marshal: libdaf.so stands alone, and the Python functions that need the module say so."""
    if importlib.util.find_spec("torch") is None:
        return MARSHAL
    made = f"torch {importlib.metadata.version('torch')}, {sys.implementation.cache_tag}"
    if os.path.exists(MARSHAL_MADE):
        with open(MARSHAL_MADE) as f:
            force = force or f.read() != made
    else:
        force = True
    if not (force or _stale(MARSHAL, [MARSHAL_SOURCE, HEADERS[-1]])):
        return MARSHAL
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    cxx = shutil.which("g++")
    if cxx is None:
        raise RuntimeError("g++ not found: the marshalling module cannot be built")
    include = [f"-I{sysconfig.get_paths()['include']}"]
    for path in [*cpp_extension.include_paths(), os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")]:
        include += ["-isystem", path]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *include,
           MARSHAL_SOURCE, "-o", MARSHAL, f"-L{libs}", "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python", "-lc10_cuda", f"-L{HERE}",
           "-l:libdaf.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on marshal.cpp:\n{r.stdout}\n{r.stderr}")
    with open(MARSHAL_MADE, "w") as f:
        f.write(made)
    return MARSHAL


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
