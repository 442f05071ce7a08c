"""Builds libblstm_mi355.so for gfx950 from csrc/ with hipcc, in-tree.

Usage: python -m paper_1904_04956_amd.build   (or build_library() from Python)
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libblstm_mi355.so")
SOURCES = ["api.hip", "gemm.hip", "gemm_f32.hip", "recurrent.hip", "recurrent_small.hip", "recurrent_tile.hip", "recurrent_multi.hip", "recurrent_f32.hip", "residency.hip", "cell.hip", "softmax.hip", "losses.hip", "losses_fused.hip", "losses_rows.hip", "update.hip", "muon.hip", "adapters.hip", "pad.hip"]

# The packed-fp32 feature is switched off for all device code on purpose.
HIPCC_FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-Wall", "-Wno-unused-function",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc(), *HIPCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    if src.startswith("recurrent"):
        cmd.append("-Rpass-analysis=kernel-resource-usage")
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    lines = [l for l in r.stderr.splitlines() if noise not in l]
    if src.startswith("recurrent"):
        # a persistent kernel whose registers spill to scratch memory is rejected: keep them resident
        name = ""
        for l in lines:
            if "Function Name:" in l:
                name = l.split("Function Name:")[1].split()[0]
            if "ScratchSize [bytes/lane]:" in l and "rec" in name:
                if int(l.split("ScratchSize [bytes/lane]:")[1].split()[0]) != 0:
                    raise RuntimeError(f"persistent kernel {name} spills to scratch memory")
        keep, skip = [], 0
        for l in lines:                      # drop the remarks and the source excerpts printed under them
            if "remark:" in l:
                skip = 2
                continue
            if skip and (l.lstrip().startswith("|") or l.lstrip()[:1].isdigit() or "^" in l):
                skip -= 1
                continue
            keep.append(l)
        lines = keep
    err = "\n".join(lines)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_library(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [hipcc(), "-shared", "--offload-arch=gfx950", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build_library()
