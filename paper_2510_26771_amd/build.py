"""Builds libstamp_hip.so (gfx950) in-tree with hipcc.  Run as `python -m paper_2510_26771_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libstamp_hip.so")

SOURCES = ["stamp_fp8_gemm.hip", "stamp_fp8_rows.hip", "stamp_fp8_quant.hip", "stamp_fp8_api.hip", "stamp_route.hip", "stamp_bottom1d_6.hip", "stamp_bottom1d_5.hip", "stamp_bottom1d_7.hip", "stamp_gemm6.hip", "stamp_gemm6_half.hip", "stamp_gemm6_pair.hip", "stamp_gemm6_hi.hip",
           "stamp_actquant.hip", "stamp_bottom1d_4.hip", "stamp_bottom1d_3.hip", "stamp_api.hip", "stamp_weight.hip", "stamp_gemm.hip", "stamp_hi6.hip", "stamp_grouped.hip", "stamp_inverse.hip", "stamp_probe.hip", "stamp_general.hip", "stamp_dct.hip", "stamp_lanes1d.hip", "stamp_lanes2d.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(len(SOURCES), 8)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB_PATH, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    if verbose:
        print(f"built {LIB_PATH}")
    return LIB_PATH


if __name__ == "__main__":
    build()
