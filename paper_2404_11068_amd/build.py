"""Build libevoattn.so (gfx950) in-tree with hipcc.

    python -m paper_2404_11068_amd.build
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libevoattn.so")
OBJDIR = os.path.join(PKG, "_build")

SOURCES = ["evo_fwd.hip", "evo_bwd.hip", "evo_bwd_qbias.hip", "evo_bwd_fused.hip", "evo_ln.hip", "evo_proj.hip", "evo_pair_bias.hip", "evo_optim.hip",
           "evo_proj_bwd.hip", "evo_pair_bias_bwd.hip", "evo_relpos.hip", "evo_muon.hip",
           "evo_probe.hip", "evo_api.cpp", "evo_ln_api.cpp", "evo_proj_api.cpp", "evo_optim_api.cpp",
           "evo_relpos_api.cpp", "evo_muon_api.cpp", "evo_graph.cpp"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 VALU instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA results straight into arch VGPRs (no accumulator-register round trip)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    # the kernels use infinities (masks, empty rows) but never NaN: without
    # this, every fmaxf first canonicalises both inputs (one extra VALU op each)
    "-fno-honor-nans",
    "-Wall", "-Wno-unused-function",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the device-only feature flag; that warning is noise
    err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build() -> str:
    """Compile every source and link the shared library; returns its path."""
    os.makedirs(OBJDIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n%s" % res.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
