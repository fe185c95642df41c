"""The learner's kernels keep everything in registers: no scratch memory, no spilled vector
registers (compiles the device code to assembly; no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2602_01665_amd import build as hip_build


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    asm = tmp_path_factory.mktemp("asm") / "tabx_learner.s"
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only"] + hip_build.LEARNER_SOURCES +
                   ["-o", str(asm)], check=True, capture_output=True)
    return asm.read_text()


def test_no_scratch_memory_and_no_spills(listing):
    kernels = re.findall(r"\.name:\s+(_ZN4tabx\w+)\n(.*?)\.wavefront_size", listing, re.S)
    assert len(kernels) >= 30
    for name, meta in kernels:
        assert re.search(r"\.private_segment_fixed_size:\s+0\b", meta), name
        assert re.search(r"\.vgpr_spill_count:\s+0\b", meta), name
    assert not re.search(r"\bscratch_(load|store)", listing)
    assert not re.search(r"\bflat_(load|store)", listing)       # every address is known to be global memory
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", listing)


def test_one_lane_per_row_needs_no_lds(listing):
    """What a lane holds of its row stays in registers (an array that is indexed by a runtime value
    is moved to LDS without a word)."""
    sizes = re.findall(r"\.amdhsa_kernel (_ZN4tabx\w+)\n\s+\.amdhsa_group_segment_fixed_size (\d+)", listing)
    rows = [(n, int(s)) for n, s in sizes if "sample_actions" in n or "log_prob" in n]
    assert len(rows) == 4 and all(s == 0 for _, s in rows), rows


def test_draws_leave_room_for_five_wavefronts(listing):
    """512 registers of a SIMD's lane, handed out in eights."""
    sizes = re.findall(r"\.amdhsa_kernel (_ZN4tabx\w*sample_actions\w+)\n(?:.*\n)*?\s+\.amdhsa_next_free_vgpr (\d+)", listing)
    assert len(sizes) == 2 and all(int(n) <= 96 for _, n in sizes), sizes
