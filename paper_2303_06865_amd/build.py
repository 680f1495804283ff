"""Build libfg.so (HIP, gfx950 only) in-tree:  python -m paper_2303_06865_amd.build"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libfg.so")

SOURCES = [
    "fg_quant.hip",
    "fg_norm.hip",
    "fg_gemm_fewrows.hip",
    "fg_gemm_fewrows_ln.hip",
    "fg_gemm_small_m.hip",
    "fg_gemm_large_m.hip",
    "fg_gemm_stream.hip",
    "fg_gemm_f16w.hip",
    "fg_gemm_f16_tiles.hip",
    "fg_attn_decode.hip",
    "fg_attn_topk.hip",
    "fg_attn_prefill.hip",
    "fg_kv_i8.hip",
    "fg_attn_i8.hip",
    "fg_beam.hip",
    "fg_layer.hip",
]

COMMON = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    # packed-FP32 instructions stay off on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]
# the quantizers must be bit-exact functions of their inputs: no fused multiply-add, IEEE division
PER_FILE = {"fg_quant.hip": ["-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt"],
            "fg_kv_i8.hip": ["-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt"]}


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    return "hipcc"


def _compile(src: str, extra=()) -> str:
    obj = os.path.join(BUILD, src.replace(".hip", ".o"))
    cmd = [_hipcc(), *COMMON, *PER_FILE.get(src, []), *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), r.stderr[-6000:]))
    return obj


def build(verbose: bool = True, jobs: int = 8, extra=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(jobs, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, extra), SOURCES))
    cmd = [_hipcc(), "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s" % r.stderr[-4000:])
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(extra=sys.argv[1:])
