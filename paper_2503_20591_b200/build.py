"""Builds libnbos.so (the CUDA library behind include/nbos.h) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libnbos.so")
SOURCES = ("nbos_api.cu", "nbos_derive.cu", "nbos_place.cu", "nbos_executor.cu", "nbos_cluster.cu", "nbos_sequential.cu", "nbos_probe.cu",
           "nbos_policy_distill.cu", "nbos_policy_balance.cu", "nbos_policy_sample.cu")
HEADERS = (os.path.join(ROOT, "include", "nbos.h"), os.path.join(ROOT, "include", "nbos_probe.h"),
           os.path.join(CSRC, "nbos_internal.h"), os.path.join(CSRC, "nbos_ptx.cuh"), os.path.join(CSRC, "nbos_sorted_chunk.cuh"), os.path.join(CSRC, "nbos_ranked_chunk.cuh"),
           os.path.join(CSRC, "nbos_policy.cuh"))
ARCH_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a"]


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; libnbos.so cannot be built")


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + list(HEADERS)
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into paper_2503_20591_b200/libnbos.so."""
    if not force and not _stale():
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc_path(), "-O3", "-std=c++17", "-lineinfo", "--threads", "0", *ARCH_FLAGS,
           "-Xcompiler", "-fPIC,-Wall,-Wextra", "-shared", "-cudart", "shared",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += ["-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libnbos.so")
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
