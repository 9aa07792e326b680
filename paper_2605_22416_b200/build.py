"""Builds libavmp.so (sm_100a) in-tree with nvcc.  Usable as `python -m paper_2605_22416_b200.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libavmp.so"
SOURCES = ["avmp_api.cu", "avmp_step.cu", "avmp_copy.cu", "avmp_noalloc.cu", "avmp_driver.cu",
           "avmp_sessions.cu", "avmp_ssm.cu", "avmp_attn.cu",
           "avmp_attn_prompt.cu", "avmp_conv.cu", "avmp_scan.cu", "avmp_rows.cu"]
HEADERS = [CSRC / "avmp_dev.cuh", CSRC / "avmp_step_body.cuh", CSRC / "avmp_mma.cuh", CSRC / "avmp_tc.cuh", CSRC / "avmp_lists.cuh",
           ROOT / "include" / "avmp.h"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "--shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
              "-cudart", "static", f"-I{ROOT / 'include'}", f"-I{CSRC}"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and Path(cand).exists():
            return cand
    raise RuntimeError("nvcc not found: the CUDA extension cannot be built")


def needs_build() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    return any(p.stat().st_mtime > t for p in [CSRC / s for s in SOURCES] + HEADERS)


def build_library(force: bool = False, verbose: bool = False) -> Path:
    if not force and not needs_build():
        return LIB
    tmp = LIB.with_suffix(f".tmp{os.getpid()}.so")
    cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-o", str(tmp),
           *[str(CSRC / s) for s in SOURCES]]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
