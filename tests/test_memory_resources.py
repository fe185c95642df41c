"""The kernels of a unit's memory keep everything in registers and LDS: no scratch memory, no spilled vector registers
(compiles the device code to assembly; no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2602_01665_amd import build as hip_build


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    asm = tmp_path_factory.mktemp("asm") / "tabx_memory.s"
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only"] + hip_build.MEMORY_SOURCES + ["-o", str(asm)], check=True,
                   capture_output=True)
    return asm.read_text()


def sizes(listing, kernel, what):
    return [(n, int(v)) for n, body in re.findall(r"\.amdhsa_kernel (_ZN4tabx\S*)\n(.*?)\.end_amdhsa_kernel", listing, re.S)
            if kernel in n for v in re.findall(rf"\.amdhsa_{what} (\d+)", body)]


def test_no_scratch_memory_and_no_spills(listing):
    kernels = re.findall(r"\.name:\s+(_ZN4tabx\w+)\n(.*?)\.wavefront_size", listing, re.S)
    assert len(kernels) >= 100
    for name, meta in kernels:
        assert re.search(r"\.private_segment_fixed_size:\s+0\b", meta), name
        assert re.search(r"\.vgpr_spill_count:\s+0\b", meta), name
    assert not re.search(r"\bscratch_(load|store)", listing)
    assert not re.search(r"\bflat_(load|store)", listing)       # every address is known to be global memory
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", listing)


def test_workgroups_fit_a_cu(listing):
    """160 KB of LDS and 512 registers of a SIMD's lane: three workgroups of 64-wide 16-bit heads, two of 128-wide ones."""
    for kernel in ("attention_kernel", "attention_grad_kernel", "attention_grad_apart_kernel"):
        lds, registers = dict(sizes(listing, kernel, "group_segment_fixed_size")), dict(sizes(listing, kernel, "next_free_vgpr"))
        assert lds and registers
        for name in lds:
            width = int(re.search(r"ILi(\d+)", name)[1])
            wide = re.search(rf"ILi{width}ELi0E", name) is not None             # f32
            workgroups = 1 if wide and width == 128 else 2 if width >= 96 or wide else 3
            if "ILi128ELi2E" in name and "apart" in name:
                workgroups = 1
            assert workgroups * lds[name] <= 160 * 1024, name
            waves = -(-workgroups * (width // 16) // 4)
            assert -(-registers[name] // 8) * 8 * waves <= 512, (name, registers[name])


def test_arguments_are_not_spilled(listing):
    """What all of an attention needs is fetched where it is needed (at the top, it would be moved to vector registers)."""
    for name, meta in re.findall(r"\.name:\s+(_ZN4tabx\d+tabx_attention_\w+)\n(.*?)\.wavefront_size", listing, re.S):
        spilled = int(re.search(r"\.sgpr_spill_count:\s+(\d+)", meta)[1])
        assert spilled <= 64, (name, spilled)


def test_a_stream_gradient_in_place_is_read_before_it_is_overwritten(listing):
    """A row of more lanes than a wavefront has its last elements read by several of them, and grad_x may lie where
    grad_sum does: behind the barrier of a row's sum, at whose other side stores begin, only the next row's loads (of the
    widest form: rstd and three arrays) may be under way."""
    seen = 0
    for m in re.finditer(r"^(_ZN4tabx\w*rms_grad_kernelI\w+):.*?\n(.*?)s_endpgm", listing, re.S | re.M):
        lanes, pieces, *_, streamed = map(int, re.search(r"ILi(\d+)ELi(\d+)ELi(\d)ELi(\d)ELb(\d)ELb(\d)", m[1]).groups())
        if lanes <= 64 or not streamed:
            continue
        seen += 1
        under_way = 1 + 3 * pieces if lanes == 1024 else 0
        sums, waited = 0, None
        for line in m[2].split("\n"):
            w = re.match(r"\s*s_waitcnt.*vmcnt\((\d+)\)", line)
            waited = int(w[1]) if w else waited
            if re.match(r"\s*s_barrier", line) and waited is not None:
                sums += 1
                assert waited <= under_way, (m[1], waited)
        assert sums, m[1]
    assert seen == 20
