"""Builds the HIP library (gfx950) in-tree: ``python -m paper_2210_07454_amd.build``."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SO = os.path.join(HERE, "libsams.so")
SOURCES = ["sams_api.hip", "sams_update.hip", "sams_sketch.hip", "sams_plan.hip", "sams_pull.hip", "sams_push.hip", "sams_select.hip", "sams_noalloc.hip",
           "sams_norm.hip", "sams_xent.hip", "sams_ortho.hip", "sams_dropout.hip", "sams_attn.hip", "sams_attn_back.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                      # formulas are evaluated as written (no fused multiply-add)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument", "-parallel-jobs=8",
]


def build(verbose: bool = False) -> str:
    cmd = [HIPCC, *FLAGS, *[os.path.join(CSRC, s) for s in SOURCES], "-o", SO]
    if verbose:
        print(" ".join(cmd), flush=True)
    p = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in p.stderr.splitlines() if "packed-fp32-ops" not in l)
    if p.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return SO


if __name__ == "__main__":
    print(build(verbose=True))
