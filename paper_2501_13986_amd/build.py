"""Builds libcgtp.so (the C-ABI library) in-tree with hipcc for gfx950.

Usage: python -m paper_2501_13986_amd.build   (also called by __graft_entry__.build()).
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcgtp.so")
SOURCES = ["api.cpp", "cg_real.cpp", "emit_uvu.cpp", "emit_uvw.cpp", "emit_uvw_ps.cpp", "emit_norm.cpp", "jit.cpp", "api_layer.cpp", "csr.hip", "gated_f32.hip", "gated_f64.hip"]
# packed fp32 instructions are disabled for every HIP translation unit of this project
DEVICE_FLAGS = ["--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build_library(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def compile_one(src: str) -> str:
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        cmd = [hipcc, "-c", "-O2", "-fPIC", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__"]
        if src.endswith(".hip"):
            cmd += ["-Wno-unused-result", os.path.join(CSRC, src), "-o", obj] + DEVICE_FLAGS
        else:   # -x must precede the input
            cmd += ["-I/opt/rocm/include", "-x", "c++", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        return obj

    # the longest first; the gated kernels take most of a minute each
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, sorted(SOURCES, key=lambda f: not f.startswith("gated"))))
    cmd = [hipcc, "-shared", "-o", LIB] + objs + ["-L/opt/rocm/lib", "-lhiprtc", "-lamd_comgr", "-lamdhip64", "-ldl",
                                                  "-Wl,-rpath,/opt/rocm/lib"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    build_library()
    sys.exit(0)
