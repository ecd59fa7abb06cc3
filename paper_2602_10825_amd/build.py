"""Builds libflowcache.so (HIP, gfx950 only) in-tree with hipcc.

    python -m paper_2602_10825_amd.build
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libflowcache.so")
SOURCES = ["api.hip", "decide.hip", "attend_f32.hip", "attend_bf16.hip", "attend_kv4.hip", "attend_kv4_f32.hip", "mass.hip",
           "compress.hip", "residual.hip", "rope.hip", "kv4.hip", "sched.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
# The attention kernels' inputs are finite by contract and they may assume so (cheaper max);
# every file that CHECKS arguments for NaN (api.hip) or writes NaN on purpose (decide, mass) is
# compiled with full NaN semantics.
NO_NAN_OK = {"attend_bf16.hip", "attend_f32.hip", "attend_kv4.hip", "attend_kv4_f32.hip"}


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    extra = ["-fno-honor-nans"] if src in NO_NAN_OK else []
    cmd = [HIPCC, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{res.stdout}\n{res.stderr}")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(6, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
    # stand-alone probe of the achievable MFMA / HBM peaks (not part of the library)
    probe = os.path.join(HERE, "peak_probe")
    cmd = [HIPCC, *FLAGS, os.path.join(CSRC, "peak_probe.hip"), "-o", probe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on peak_probe.hip:\n{res.stdout}\n{res.stderr}")
    if verbose:
        print(f"built {LIB} and {probe}")
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
