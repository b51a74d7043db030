"""Builds libciera.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libciera.so")
SOURCES = ["ciera_host.cu", "ciera_encode.cu", "ciera_encode_hashed.cu", "ciera_decode.cu", "ciera_entropy.cu", "ciera_kernels.cu",
           "ciera_route.cu", "ciera_experts.cu", "ciera_fp8.cu", "ciera_fp8_product.cu", "ciera_fp4.cu", "ciera_fp4_product.cu",
           "ciera_tokens.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
    "-Xptxas", "-v",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "ciera.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    tmp = f"{LIB}.{os.getpid()}.tmp"  # built beside its place and moved there whole: nobody loads half a library
    with tempfile.TemporaryDirectory() as work:
        objects = [os.path.join(work, s + ".o") for s in SOURCES]
        include = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
        steps = [[_nvcc(), "-c", "-o", o] + include + NVCC_FLAGS + [os.path.join(CSRC, s)] for s, o in zip(SOURCES, objects)]
        with ThreadPoolExecutor(min(len(steps), os.cpu_count() or 1)) as pool:  # the files side by side
            done = list(pool.map(lambda cmd: subprocess.run(cmd, capture_output=True, text=True), steps))
        if all(r.returncode == 0 for r in done):
            done.append(subprocess.run([_nvcc(), "-shared", "-o", tmp] + NVCC_FLAGS + objects, capture_output=True, text=True))
    for r in done:
        if verbose or r.returncode != 0:
            print(r.stdout)
            print(r.stderr)
    if any(r.returncode != 0 for r in done):
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError("nvcc failed building libciera.so")
    os.replace(tmp, LIB)
    return LIB


def ensure_library(wait_s: float = 600.0) -> str:
    """Builds the library if it is not there at all (a fresh checkout); a library that is there is used as it
    is.  Of several processes started together (one per GPU) the one with LOCAL_RANK 0 builds, the others wait."""
    import time

    if os.path.exists(LIB):
        return LIB
    if int(os.environ.get("LOCAL_RANK", "0")) == 0:
        return build_library(force=True)
    t0 = time.time()
    while not os.path.exists(LIB):
        if time.time() - t0 > wait_s:
            raise RuntimeError("libciera.so did not appear: build it with python -m paper_2609_04609_b200.build")
        time.sleep(1.0)
    return LIB


if __name__ == "__main__":
    build_library(force=True, verbose=True)
