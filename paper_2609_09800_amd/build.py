"""Build ``libhbf.so`` (HIP for gfx950) in-tree with hipcc.

Usage: ``python -m paper_2609_09800_amd.build``.  Always recompiles.
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhbf.so")
SOURCES = ["hbf_api.cpp", "hbf_kernels.hip", "hbf_gemv.hip", "hbf_cache.hip", "hbf_blocking.hip", "hbf_vmem.hip",
           "hbf_layers.hip", "hbf_small.hip", "hbf_cache_chunk.hip", "hbf_ops_api.cpp", "hbf_kv.hip", "hbf_attn.hip", "hbf_moe.hip"]
ARCH = "gfx950"

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", f"--offload-arch={ARCH}",
    # packed-FP32 instructions stay off (hipcc -O3 would otherwise form them)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    "-Wall", "-Wno-unused-result", "-Wno-unused-variable",
]


def build(verbose=False):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    srcs = []
    for s in SOURCES:
        p = os.path.join(CSRC, s)
        srcs.append(p)
    tmp = LIB + ".tmp"
    cmd = [hipcc] + FLAGS + srcs + ["-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("hipcc failed building libhbf.so")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
