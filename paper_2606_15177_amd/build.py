"""Builds the gfx950 shared library of the MoE-layer hot path in-tree.

    python -m paper_2606_15177_amd.build

Compiles every ``csrc/*.hip`` with hipcc for gfx950 (one process per file)
and links ``libmoe_gfx950.so`` next to this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB_NAME = "libmoe_gfx950.so"
LIB_PATH = os.path.join(HERE, LIB_NAME)
ARCH = "gfx950"

SOURCES = ["route.hip", "permute.hip", "combine.hip", "ffn_skinny.hip", "ffn_mid.hip", "ffn_tiled.hip", "place.hip", "window.hip",
           "moe_abi.hip"]
# the 8-bit experts
SOURCES_I8 = ["quant.hip", "gemm_i8.hip", "i8_few.hip", "i8_mid.hip", "i8_tiled.hip"]
# the experts in 8-bit floating point, and the norms around the layer
SOURCES_F8 = ["quant_f8.hip", "gemm_f8.hip", "f8_few.hip", "f8_mid.hip", "f8_tiled.hip", "norm.hip"]

CXXFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # code object v5 loads on every ROCm runtime this library may meet (torch bundles its own)
    "-mcode-object-version=5",
    # packed fp32 VALU ops stay off (the compiler would otherwise form them)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


# matrix instructions write ordinary registers, where the e4m3 products' scaled
# additions read them (accumulation registers cost a move each)
EXTRA_FLAGS = {s: ["-mllvm", "-amdgpu-mfma-vgpr-form"] for s in ("f8_few.hip", "f8_mid.hip", "f8_tiled.hip")}


def _hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cand = os.path.join(rocm, "bin", "hipcc")
    return cand if os.path.exists(cand) else "hipcc"


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc(), *CXXFLAGS, *EXTRA_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def _check_resolved(lib: str) -> None:
    """A shared library links even when one of its own functions was never
    emitted (the loader would only fail later); reject undefined symbols of
    the library's namespace."""
    r = subprocess.run(["nm", "-D", "--undefined-only", lib], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nm failed on {lib}:\n{r.stderr}")
    missing = [ln.split()[-1] for ln in r.stdout.splitlines() if "_ZN3moe" in ln]
    if missing:
        os.remove(lib)
        raise RuntimeError("library references undefined symbols of its own: " + ", ".join(missing))


def build(verbose: bool = False) -> str:
    """Compile and link the library; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    sources = SOURCES + SOURCES_I8 + SOURCES_F8
    with cf.ThreadPoolExecutor(max_workers=min(len(sources), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, sources))
    tmp = LIB_PATH + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    _check_resolved(tmp)
    os.replace(tmp, LIB_PATH)
    if verbose:
        print(f"built {LIB_PATH}")
    return LIB_PATH


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
