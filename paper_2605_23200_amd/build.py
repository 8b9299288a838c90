"""Builds the HIP library behind include/ams.h for gfx950 into paper_2605_23200_amd/libams.so."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libams.so")
OBJ_DIR = os.path.join(PKG, "_build")

SOURCES = ["ams_api.hip", "score.hip", "score_causal.hip", "score_last.hip", "score_causal_last.hip", "score_keys.hip", "score_park.hip", "score_unit.hip", "mass_segment.hip", "select.hip", "compact.hip",
           "cache_api.hip", "append.hip", "attend.hip", "recode.hip", "evict.hip"]

# -ffp-contract=off: multiply-adds are fused only where the source says fmaf(), so that host-checkable
# double arithmetic (quotas, normalisers) rounds exactly like plain C.
# Packed fp32 instructions are switched off: some of their forms have given wrong results on the machines used.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(src):
    obj = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(jobs: int = 6) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, SOURCES))
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    return LIB


if __name__ == "__main__":
    print(build())
