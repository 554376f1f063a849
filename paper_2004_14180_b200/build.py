"""Builds paper_2004_14180_b200/libqadam.so from csrc/ with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libqadam.so")
SOURCES = [os.path.join(CSRC, "qadam_api.cu"), os.path.join(CSRC, "qadam_noalloc.cu"), os.path.join(CSRC, "qadam_norm.cu"),
           os.path.join(CSRC, "qadam_adamw.cu"), os.path.join(CSRC, "qadam_embedding.cu"),
           os.path.join(CSRC, "qadam_layer.cu"), os.path.join(CSRC, "qadam_product.cu")]
HEADERS = [os.path.join(CSRC, "qadam_device.cuh"), os.path.join(CSRC, "qadam_kernels.cuh"),
           os.path.join(CSRC, "qadam_server_pipe.cuh"),
           os.path.join(CSRC, "qadam_worker_resident.cuh"), os.path.join(CSRC, "qadam_worker_stream.cuh"),
           os.path.join(CSRC, "qadam_host.h"), os.path.join(CSRC, "qadam_tensors.cuh"),
           os.path.join(CSRC, "qadam_rows.cuh"),
           os.path.join(_ROOT, "include", "qadam.h")]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    # IEEE arithmetic everywhere: no FMA contraction, exact division and root, subnormals kept
    "--fmad=false", "--prec-div=true", "--prec-sqrt=true", "--ftz=false",
    "-Xcompiler", "-fPIC",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    flags = NVCC_FLAGS + ["-I", os.path.join(_ROOT, "include"), "-I", CSRC] + (["-Xptxas", "-v"] if verbose else [])
    with tempfile.TemporaryDirectory() as work:           # the sources at the same time, then one library of their objects
        def compile_one(source: str) -> str:
            target = os.path.join(work, os.path.basename(source) + ".o")
            subprocess.run([_nvcc()] + flags + ["-c", "-o", target, source], check=True)
            return target
        with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
            objects = list(pool.map(compile_one, SOURCES))
        subprocess.run([_nvcc()] + NVCC_FLAGS + ["-shared", "-o", LIB] + objects, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
