"""In-tree build of libakv.so (nvcc, sm_103a only)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libakv.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
          "-I", CSRC]
SOURCES = {
    "akv_api.cpp": [],
    "akv_decode.cu": [],
    "akv_decode_g1.cu": [],  # the decode kernels per query-group size, compiled in parallel
    "akv_decode_g2.cu": [],
    "akv_decode_g4.cu": [],
    "akv_decode_g8.cu": [],
    "akv_decode_g1w.cu": [],  # with more weight rows than staged rows
    "akv_decode_g2w.cu": [],
    "akv_decode_g4w.cu": [],
    "akv_decode_g8w.cu": [],
    "akv_paged_api.cpp": [],
    "akv_paged_append.cu": [],
    "akv_paged_attn.cu": [],
    "akv_paged_evict.cu": [],
    "akv_paged_query.cu": [],
    "akv_paged_select.cu": [],
    "akv_paged_shared.cu": [],
    "akv_paged_weights.cu": [],
    "akv_pages.cu": [],
    "akv_encode.cu": ["--fmad=false"],  # fp64 decisions: no contraction
}


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _compile(src: str, extra: list, verbose: bool) -> str:
    obj = os.path.join(BUILD, src + ".o")
    path = os.path.join(CSRC, src)
    deps = [path, os.path.join(ROOT, "include", "akv.h")]
    deps += [os.path.join(CSRC, h) for h in ("akv_internal.h", "akv_device.cuh", "akv_decode.cuh", "akv_paged.cuh", "akv_paged_tc.cuh")]
    if os.path.exists(obj) and all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in deps):
        return obj
    cmd = [_nvcc(), *ARCH, *COMMON, *extra, "-c", path, "-o", obj]
    if src.endswith(".cpp"):
        cmd = [_nvcc(), *COMMON, "-x", "c++", "-c", path, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda kv: _compile(kv[0], kv[1], verbose), SOURCES.items()))
    if not os.path.exists(LIB) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        tmp = LIB + f".tmp{os.getpid()}"
        cmd = [_nvcc(), *ARCH, "-shared", "-o", tmp, *objs]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
