"""Builds the HIP library in-tree: paper_2502_11490_amd/libgmpgr_ann.so (gfx950 only)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgmpgr_ann.so")
SOURCES = ["api.hip", "search_kernels.hip", "search_fused.hip", "search_wave.hip", "mlp_alu.hip", "mlp_any.hip", "mlp_mfma.hip", "mlp_mfma_stream.hip", "mlp_mfma_f8.hip", "noise.hip", "noalloc.hip",
           "brute_force.hip", "rows.hip", "layer_norm.hip", "dropout.hip", "gated_ffn.hip", "ffn_bf16.hip", "ffn_f16.hip", "ffn_f32.hip", "ffn_few.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc] + FLAGS + [os.path.join(CSRC, s) for s in SOURCES] + ["-o", LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed:\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
