"""Builds libscalecom.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libscalecom.so")
STAMP = LIB + ".srchash"

SOURCES = ["scalecom.cu", "topk_static.cu", "operators.cu"]
HEADERS = ["common.cuh", "topk_select.cuh", "learner_pass.cuh", "chunk_select.cuh", "diagnostics.cuh", "exchange.cuh", "layer_topk.cuh", "small_step.cuh",
           "ops_common.cuh", "ffn_tokens.cuh", "layer_norm.cuh", "ns_small.cuh", "operand_prep.cuh", "tc_product.cuh"]
API_HEADERS = ["scalecom.h", "scalecom_operators.h"]

NVCC_FLAGS = [
    "-O3", "-std=c++17",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-lineinfo",
    "-Xcompiler", "-fPIC", "-shared",
    "-cudart", "static", "--threads", "4",
]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: cannot build libscalecom.so")
    return exe


def source_hash() -> str:
    h = hashlib.sha256(" ".join(NVCC_FLAGS).encode())
    for name in SOURCES + HEADERS:
        with open(os.path.join(CSRC, name), "rb") as f:
            h.update(f.read())
    for name in API_HEADERS:
        with open(os.path.join(INCLUDE, name), "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def is_current() -> bool:
    if not (os.path.exists(LIB) and os.path.exists(STAMP)):
        return False
    with open(STAMP) as f:
        return f.read().strip() == source_hash()


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile if the library is missing or its sources changed; returns the library path."""
    if not force and is_current():
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
           *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
    subprocess.run(cmd, check=True, cwd=HERE)
    os.replace(tmp, LIB)
    with open(STAMP, "w") as f:
        f.write(source_hash())
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
