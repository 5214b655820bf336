"""Builds libsketchwalk.so (gfx950) in-tree from csrc/*.hip with hipcc, and the
host module _host_q8.so from csrc/host_q8.cpp with g++.

Usage: python -m paper_2602_07397_amd.build   (or build() from Python)
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJDIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsketchwalk.so")
HOST = os.path.join(HERE, "_host_q8.so")
ARCH = "gfx950"

# Packed-fp32 instructions are disabled for all device code: hipcc -O3 would
# otherwise form v_pk_* fp32 ops from ordinary float code.
HIPFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]

# Per-source extras. The prefill attention kernel post-processes its score
# MFMA results on the VALU and runs two wavefronts per SIMD within 256
# registers each: the VGPR form of the MFMA instructions keeps accumulators in
# VGPRs, so no AGPR-to-VGPR copies are needed. The 8-bit decode attention runs
# three wavefronts per SIMD that way instead of two.
EXTRA = {
    "attn_prefill.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "attn_decode_q8.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
}


def _hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm toolchain required)")


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    cmd = [_hipcc(), *HIPFLAGS, *EXTRA.get(os.path.basename(src), []), "-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{res.stderr}")
    return obj


def _build_host() -> None:
    """The CPython module that marshals the 8-bit cache's calls (host code only)."""
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    dirs = [*include_paths(), sysconfig.get_paths()["include"]]
    libs = library_paths()[0]
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-isystem{d}" for d in dirs), os.path.join(CSRC, "host_q8.cpp"), "-o", HOST + ".tmp",
           f"-L{libs}", f"-Wl,-rpath,{libs}", "-ltorch_python", "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"g++ failed for host_q8.cpp:\n{res.stderr}")
    os.replace(HOST + ".tmp", HOST)


def build(verbose: bool = False) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    srcs = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))
    jobs = min(len(srcs), max(1, min(16, os.cpu_count() or 1)))
    with concurrent.futures.ThreadPoolExecutor(max_workers=jobs + 1) as ex:
        host = ex.submit(_build_host)
        objs = list(ex.map(_compile, srcs))
        host.result()
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
