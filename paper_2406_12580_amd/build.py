"""Build librecblr.so (the HIP kernels and the C ABI) for gfx950, in-tree.

    python -m paper_2406_12580_amd.build        # or: python paper_2406_12580_amd/build.py

Every source is compiled with hipcc for gfx950 only, with packed-fp32
instructions disabled, and linked into paper_2406_12580_amd/librecblr.so.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "librecblr.so")
SOURCES = ["capi.cpp", "scan_fwd.hip", "scan_bwd.hip", "step.hip", "gemm.hip", "ablation.hip",
           "gated.hip", "model.hip", "noalloc.hip", "fused_fwd.hip", "fused_bwd.hip",
           "proj_bwd.hip", "ffn.hip", "head.hip", "capi_ops.cpp", "adamw.hip", "sample.hip",
           "delta_step.hip", "delta_fwd.hip", "delta_bwd.hip",
           "delta_split.hip", "embed.hip", "qk_norm.hip", "policy.hip", "muon.hip"]
# Linear layers that the matrix-core tiles do not take go to rocBLAS.
LIBS = ["-L/opt/rocm/lib", "-lrocblas"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]
# -O3 unswitches the delta rule's gradient kernel on its waves' roles into copies that spill
# (587 registers of the fp32 one at 64 columns); -O2 keeps it within its registers for keys of up
# to 64, and at 92 to 160 registers in scratch memory beyond.
OPT = {"delta_bwd.hip": "-O2"}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    flags = [OPT.get(src, f) if f == "-O3" else f for f in FLAGS]
    cmd = [HIPCC, *flags, "-c", os.path.join(CSRC, src), "-o", obj]
    if src.endswith(".hip"):
        cmd[1:1] = ["-x", "hip"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{res.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source (always) and link librecblr.so; returns its path."""
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, *LIBS, "-o", tmp]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
