"""Compile the HIP sources into paper_2506_10470_amd/libtdp.so (gfx950 only) and the host-only
scheduler into paper_2506_10470_amd/libtdp_sched.so.

hipcc cross-compiles without a GPU.  Objects go to paper_2506_10470_amd/_build/ (git-ignored);
the shared library stays in-tree so that it travels with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libtdp.so")
SCHED_LIB = os.path.join(HERE, "libtdp_sched.so")
SOURCES = ("gemm.hip", "gemm_int.hip", "gemm_stats.hip", "attention.hip", "elementwise.hip", "stage.hip", "probe.hip",
           "gemm_static.hip", "linear_i8.hip", "logprob.hip")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass warns that it does not know the packed-fp32 feature: harmless
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("command failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, err))
    if err.strip():
        sys.stderr.write(err + "\n")


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    jobs = []
    for src in SOURCES:
        obj = os.path.join(BUILD, src.replace(".hip", ".o"))
        objs.append(obj)
        jobs.append([hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    with ThreadPoolExecutor(max_workers=8) as ex:
        list(ex.map(_run, jobs))
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB])
    cxx = os.environ.get("CXX", "g++")
    _run([cxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-Wextra",
          os.path.join(CSRC, "sched.cpp"), "-o", SCHED_LIB])
    if verbose:
        print("built", LIB)
        print("built", SCHED_LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
