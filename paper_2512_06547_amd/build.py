"""Builds liba3po.so (HIP, gfx950 only) in-tree with hipcc, and the binding's look at lists of tensors with the host compiler."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "liba3po.so")
TENSORS = os.path.join(PKG, "a3po_tensors.so")  # against PyTorch's headers; loaded by the binding alone
SOURCES = ["a3po_api.hip", "a3po_rows.hip", "a3po_few.hip", "a3po_tokens.hip", "a3po_shard.hip", "a3po_gemm.hip", "a3po_lmhead.hip",
           "a3po_lmhead_bwd.hip", "a3po_norm.hip", "a3po_adjust.hip", "a3po_w4.hip", "a3po_sample.hip", "a3po_adamw.hip", "a3po_w4_quantize.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# packed fp32 VALU forms are switched off for every device translation unit
# (the atomic optimizer would turn the row queue's one-lane atomic into a wave-wide scan that
# needs its result at once; the plain atomic lets the claim stay in flight behind the row's loads)
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def _newest(paths) -> float:
    return max(os.path.getmtime(p) for p in paths)


def _stale(so: str, paths) -> bool:
    return not os.path.exists(so) or os.path.getmtime(so) < _newest(paths)


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    subprocess.check_call([HIPCC, *FLAGS, "-c", src, "-o", obj])
    return obj


def _compile_tensors() -> None:
    import sysconfig

    import torch
    at = os.path.dirname(torch.__file__)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
                           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, "-I", os.path.join(at, "include"),
                           "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"),
                           "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "a3po_tensors.cpp"), "-o", TENSORS,
                           "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])


def _try_tensors() -> None:
    """The library does not depend on it: without PyTorch's headers or a host compiler only those two calls of the binding are missing."""
    try:
        _compile_tensors()
    except (ImportError, OSError, subprocess.CalledProcessError) as why:
        if os.path.exists(TENSORS):
            os.remove(TENSORS)
        print(f"{os.path.basename(TENSORS)} was not built ({why}): the binding's adamw_step and grad_norm will raise", file=sys.stderr)


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every kernel file and link liba3po.so, and a3po_tensors.so where that can be.  force=False skips what is up to date."""
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")] + [os.path.join(ROOT, "include", "a3po.h")]
    library = force or _stale(LIB, sources() + headers)
    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        tensors = ex.submit(_try_tensors) if force or _stale(TENSORS, [os.path.join(CSRC, "a3po_tensors.cpp")]) else None
        if library:
            os.makedirs(OBJ, exist_ok=True)
            objs = list(ex.map(_compile, sources()))
            subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs])
        if tensors:
            tensors.result()
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(force=True, verbose=True)
