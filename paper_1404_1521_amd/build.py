"""Builds libpolyglot.so (the HIP library behind include/polyglot.h) in-tree.

hipcc compiles every kernel for gfx950 only.  Packed-FP32 instruction
selection is switched off for all device code.
"""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libpolyglot.so")
SOURCES = ["kernels.hip", "api.hip", "operators.hip", "recurrence.hip", "operators_api.hip",
           "selective_grad_f32.hip", "selective_grad_bf16.hip", "selective_grad_f16.hip",
           "selective.hip", "convolution.hip", "beam.hip", "layers_api.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result",
]


def _run(cmd: list[str], verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{res.stderr[-8000:]}")


def build(verbose: bool = False) -> str:
    """Compiles the sources into LIB, side by side (always recompiles).  Returns LIB."""
    include = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    with tempfile.TemporaryDirectory() as objects, \
            ThreadPoolExecutor(len(SOURCES)) as pool:
        outs = [os.path.join(objects, s + ".o") for s in SOURCES]
        list(pool.map(lambda so: _run([HIPCC, *FLAGS, *include, "-c", os.path.join(CSRC, so[0]),
                                       "-o", so[1]], verbose), zip(SOURCES, outs)))
        tmp = LIB + ".tmp"
        _run([HIPCC, "-shared", "--offload-arch=gfx950", *outs, "-o", tmp], verbose)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
