"""Build libdensenet.so (HIP for gfx950) in-tree with hipcc, and libprobe.so, the matrix-core rate
probe that only the benchmark's ceiling measurement loads (not part of the descriptor path).

Every HIP source is compiled with packed-fp32 instructions disabled (hipcc otherwise forms
v_pk_*_f32 from ordinary float code).  Objects go to _build/ at the repository root.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libdensenet.so")
HEAD = os.path.join(PKG, "head")   # the head's operators: sources of their own beside the descriptor path's
SOURCES = ("plan.cpp", "api.cpp", "trace.cpp", "pyramid.hip", "conv.hip", "lrn_pool.hip", "regions.hip", "windows.hip",
           *(os.path.join(HEAD, f) for f in ("head_api.cpp", "norm.hip", "loss.hip", "adamw.hip", "blocks.hip", "scores.hip", "muon.hip")))
PROBE_SRC = os.path.join(PKG, "probe", "probe_mfma.hip")
PROBE_LIB = os.path.join(PKG, "libprobe.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-I", INCLUDE, "-I", CSRC,
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(os.path.basename(src))[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES) + 1, os.cpu_count() or 4)) as ex:
        objs = list(ex.map(_compile, SOURCES + (PROBE_SRC,)))
    for lib, parts in ((LIB, objs[:-1]), (PROBE_LIB, objs[-1:])):
        tmp = lib + ".tmp"
        cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *parts, "-o", tmp]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed for {os.path.basename(lib)}:\n{r.stderr}")
        os.replace(tmp, lib)
        if verbose:
            print(f"built {lib}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
