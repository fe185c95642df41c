"""Builds libtabx.so (the HIP library) in-tree for gfx950."""
from __future__ import annotations

import os
import subprocess
import sys

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
SOURCES = [os.path.join(_PKG, "csrc", "tabx_kernels.hip")]              # the tick
LEARNER_SOURCES = [os.path.join(_PKG, "csrc", "tabx_learner.hip")]      # the learner's side of it
MEMORY_SOURCES = [os.path.join(_PKG, "csrc", "tabx_memory.hip")]        # a unit's memory over its ticks
HEADERS = [os.path.join(_ROOT, "include", "tabx.h")] + [
    os.path.join(_PKG, "csrc", h)
    for h in ("tabx_device.h", "tabx_policy.h", "tabx_step.h", "tabx_observe.h",
              "tabx_observe_packed.h", "tabx_rows.h", "tabx_teams.h", "tabx_host.h", "tabx_norm.h",
              "tabx_sample.h", "tabx_levels.h", "tabx_rms.h", "tabx_rotary.h", "tabx_attention.h")]
LIB_PATH = os.path.join(_PKG, "libtabx.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                      # one rounding per written operation
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
    "-I", os.path.join(_ROOT, "include"),
]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc] + HIPCC_FLAGS + SOURCES + LEARNER_SOURCES + MEMORY_SOURCES + ["-o", LIB_PATH]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return LIB_PATH


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(f) > t for f in SOURCES + LEARNER_SOURCES + MEMORY_SOURCES + HEADERS)


if __name__ == "__main__":
    build(verbose=True)
    print(LIB_PATH)
    sys.exit(0)
