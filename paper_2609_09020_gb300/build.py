"""Compiles the CUDA decoder into ``_build/libpic_gb300.so`` (sm_103a only).

Each translation unit is compiled by its own nvcc process, in parallel, then
linked into one shared library with the C ABI of include/pic_decode.h,
include/pic_izpr.h, include/pic_idct.h, include/pic_fuse.h,
include/pic_huffman.h, include/pic_linear.h, include/pic_clip.h,
include/pic_group.h, include/pic_orth.h and include/pic_measure.h.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libpic_gb300.so")
SOURCES = ["pic_decode.cu", "k_fp32.cu", "k_fp32_any.cu", "k_fp32_sweep.cu", "k_tc.cu",
           "k_tc_tma.cu", "k_march.cu", "k_march_f32lat.cu", "k_strip.cu", "k_izpr.cu",
           "k_idct.cu", "k_fuse.cu", "k_huffman.cu", "k_peak.cu", "pic_linear.cu",
           "k_linear_grad.cu", "k_linear_tc.cu", "k_linear_tc_f16.cu",
           "k_linear_tc_bf16.cu", "k_linear_reg.cu",
           "k_linear_planes.cu", "k_linear_narrow.cu", "k_linear_few.cu", "k_linear_few32.cu",
           "k_linear_thin.cu", "k_linear_thin_f16.cu", "k_linear_thin_bf16.cu",
           "k_linear_thin_f32.cu",
           "k_linear_outer.cu", "k_clip.cu", "pic_group.cu", "k_group_any.cu",
           "k_group_grad.cu", "k_group_tc.cu", "k_group_tc_f16.cu", "k_group_tc_bf16.cu", "k_group_planes.cu", "k_group_few.cu",
           "k_group_thin_f16.cu", "k_group_thin_bf16.cu", "k_group_thin_f32.cu",
           "k_orth.cu", "k_orth_tc.cu", "k_orth_small.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
         "--expt-relaxed-constexpr", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    return "nvcc"


def _deps():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    files += [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    files.append(os.path.abspath(__file__))
    return files


def up_to_date() -> bool:
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(f) <= t for f in _deps())


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    """Builds the library if any source is newer than it; returns its path."""
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    extra = ["-Xptxas", "-v"] if ptxas_info else []

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        cmd = [nvcc, *ARCH, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        return obj, r.stderr

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        results = list(ex.map(compile_one, SOURCES))
    if verbose or ptxas_info:
        for _, err in results:
            sys.stderr.write(err)
    objs = [o for o, _ in results]
    tmp = LIB + ".tmp"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, ptxas_info="-v" in sys.argv))
