"""Builds libdynlayer.so (HIP kernels + C-ABI) for gfx950 in-tree with hipcc.

    python -m paper_2605_21603_amd.build
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdynlayer.so")
SOURCES = ["dynlayer.cpp", "dynsched.cpp", "dyntune.cpp", "kernels_elementwise.hip", "kernels_gemm.hip", "kernels_gemm_wide.hip", "kernels_gemm_f32.hip", "kernels_gemm_rows.hip", "kernels_attn_generic.hip",
           "kernels_attn_mfma.hip", "kernels_attn_plan.hip", "kernels_attn_prefill.hip", "kernels_moe.hip", "dynpages.cpp", "kernels_pages.hip", "dynattn.cpp", "kernels_attn_shared.hip",
           "kernels_attn_shared_plan.hip"]
# packed fp32 instructions are switched off for every kernel (hipcc flag, device pass only)
FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-x", "hip"]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    build_dir = os.path.join(HERE, "_build")
    os.makedirs(build_dir, exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(build_dir, os.path.splitext(src)[0] + ".o")
        objs.append(obj)
        cmd = [hipcc] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            raise RuntimeError("hipcc failed: %s\n%s" % (" ".join(cmd), out))
        if verbose and out.strip():
            print(out)
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
