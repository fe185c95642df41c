"""Builds libtabx.so (the HIP library) in-tree for gfx950."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

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
    with tempfile.TemporaryDirectory() as tmp:     # the sources side by side, then one library of their objects
        running = []
        for source in SOURCES + LEARNER_SOURCES + MEMORY_SOURCES:
            to = os.path.join(tmp, os.path.basename(source) + ".o")
            cmd = [hipcc] + [f for f in HIPCC_FLAGS if f != "-shared"] + ["-c", source, "-o", to]
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append((cmd, to, subprocess.Popen(cmd)))
        failed = [cmd for cmd, _, p in running if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.run([hipcc] + HIPCC_FLAGS + [to for _, to, _ in running] + ["-o", LIB_PATH], check=True)
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
