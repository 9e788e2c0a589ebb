"""Builds libodsgd.so (sm_100a) in-tree with nvcc.  `python -m paper_2005_06728_b200.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from typing import List, Optional, Sequence

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libodsgd.so")
SOURCES = [os.path.join(CSRC, f) for f in ("odsgd.cu", "odsgd_lm.cu", "odsgd_gated.cu", "odsgd_dropout.cu", "odsgd_verify.cu")]
HEADERS = [os.path.join(CSRC, f) for f in ("odsgd_kernels.cuh", "odsgd_lm_host.h", "odsgd_lm_elements.cuh", "odsgd_lm_softmax.cuh",
                                           "odsgd_lm_kernels.cuh", "odsgd_gated_kernels.cuh", "odsgd_dropout_kernels.cuh",
                                           "odsgd_verify_kernels.cuh")] + [os.path.join(INCLUDE, "odsgd.h")]

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-lineinfo",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-Xcompiler", "-fPIC", "-shared", "--threads", "0",
]


def nvcc_path() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return cand


def is_stale(out: str = LIB) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS)


def build(force: bool = False, extra_flags: Optional[Sequence[str]] = None, out: str = LIB,
          verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; return its path."""
    if not force and not extra_flags and not is_stale(out):
        return out
    cmd: List[str] = [nvcc_path(), *NVCC_FLAGS, f"-I{INCLUDE}", f"-I{CSRC}"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += list(extra_flags or [])
    tmp = out + f".tmp{os.getpid()}"
    cmd += ["-o", tmp, *SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
