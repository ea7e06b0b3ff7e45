"""Build ``libbns.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIBRARY = os.path.join(HERE, "libbns.so")
SOURCES = [os.path.join(CSRC, name) for name in ("bns_api.cu", "bns_lm_api.cu", "bns_lm_step_api.cu")]
HEADERS = [os.path.join(CSRC, name) for name in (
    "bns_host.h", "bns_lm_host.h", "bns_elements.cuh", "bns_async.cuh", "bns_logits.cuh", "bns_kernels.cuh", "bns_nhwc_kernels.cuh", "bns_slab_kernels.cuh",
    "bns_rms_kernels.cuh", "bns_head_kernels.cuh", "bns_head_few_kernels.cuh", "bns_distill_kernels.cuh", "bns_logp_kernels.cuh",
    "bns_rotary_kernels.cuh", "bns_clip_kernels.cuh")] + [os.path.join(ROOT, "include", "bns.h")]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-lineinfo", "-std=c++17",
    "-Xcompiler", "-fPIC", "-shared", "--threads", "0",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def is_stale() -> bool:
    if not os.path.exists(LIBRARY):
        return True
    built = os.path.getmtime(LIBRARY)
    return any(os.path.getmtime(p) > built for p in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile if the library is missing or older than its sources; return its path."""
    if not force and not is_stale():
        return LIBRARY
    tmp = LIBRARY + f".tmp{os.getpid()}"
    cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-o", tmp, *SOURCES]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIBRARY)
    return LIBRARY


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
