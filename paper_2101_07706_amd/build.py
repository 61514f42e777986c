"""Builds libcsgs.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcsgs.so")
SOURCES = ["probs.hip", "sample.hip", "aggregate.hip", "gemm.hip", "fused.hip", "profile.hip", "digits.hip",
           "embed.hip", "residual.hip", "clip.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _hipcc(args) -> str:
    res = subprocess.run(["hipcc"] + args, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    return out


def build_library(verbose: bool = False) -> str:
    """Compiles every source (several at a time) and links them."""
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        jobs = [FLAGS + ["-c", "-o", o, os.path.join(CSRC, s)] for s, o in zip(SOURCES, objects)]
        workers = max(1, min(len(jobs), int(os.environ.get("MAX_JOBS") or 0) or len(os.sched_getaffinity(0)), 8))
        with ThreadPoolExecutor(workers) as pool:
            out = list(pool.map(_hipcc, jobs))
        out.append(_hipcc(["--offload-arch=gfx950", "-shared", "-o", LIB] + objects))
    if verbose and any(o.strip() for o in out):
        print("\n".join(o for o in out if o.strip()))
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
