"""Builds ``libgs.so`` (HIP, gfx950) in-tree with hipcc.

``python -m paper_2407_15452_amd.build`` compiles every ``csrc/*.hip`` file and
links them into ``paper_2407_15452_amd/libgs.so``.  hipcc cross-compiles, so no
GPU is needed to build.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libgs.so")
OBJ_DIR = os.path.join(_HERE, "_build")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wextra",
    "-munsafe-fp-atomics",
    "-Werror=pass-failed",          # a kernel that cannot hold the occupancy it is bounded to
    # packed fp32 arithmetic is kept off for every kernel of this library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


# Files whose kernels take sampling decisions that must match the CPU reference bit for bit
# (one multiply, one compare per decision): no fused multiply-add may ever be formed there.
# sgns.hip keeps contraction on (its only bit-exact part, the negative draws, is a compare).
# choose.hip sorts scores into steps in several kernels, which have to agree; beam.hip computes a log-probability in two passes.
NO_CONTRACTION = {"walk.hip", "pairs_negs.hip", "alias_build.hip", "csr_build.hip", "choose.hip", "beam.hip"}


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found; libgs.so cannot be built")
    return exe


def _compile(src: str) -> str:
    obj = os.path.join(OBJ_DIR, os.path.basename(src) + ".o")
    extra = ["-ffp-contract=off"] if os.path.basename(src) in NO_CONTRACTION else []
    cmd = [hipcc(), *HIPCC_FLAGS, *extra, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops' is not a recognized feature"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_lib(jobs: int = 8) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, sources))
    subprocess.run([hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs],
                   check=True)
    return LIB


if __name__ == "__main__":
    print(build_lib())
