"""The structs and constants of a unit's memory as a C compiler lays them out, against the Python binding's
(no GPU needed)."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <stddef.h>
#include <stdio.h>
#include "tabx.h"
#define FIELD(s, f) printf(#s "." #f " %zu %zu\n", offsetof(s, f), sizeof(((s *)0)->f))
#define VALUE(v) printf(#v " %lld 0\n", (long long)(v))
int main(void)
{
    VALUE(sizeof(TabxHeads)); VALUE(sizeof(TabxAxis));
    FIELD(TabxHeads, data); FIELD(TabxHeads, tick_stride); FIELD(TabxHeads, row_stride); FIELD(TabxHeads, head_stride);
    FIELD(TabxHeads, type);
    FIELD(TabxAxis, position); FIELD(TabxAxis, type); FIELD(TabxAxis, units); FIELD(TabxAxis, pairs);
    VALUE(TABX_F32); VALUE(TABX_BF16); VALUE(TABX_F16); VALUE(TABX_E4M3); VALUE(TABX_I32);
    VALUE(TABX_ROTARY_MAX_WIDTH); VALUE(TABX_ROTARY_MAX_AXES); VALUE(TABX_ATTENTION_MAX_WIDTH); VALUE(TABX_ATTENTION_MAX_HEADS);
    return 0;
}
"""


@pytest.fixture(scope="module")
def laid_out(tmp_path_factory):
    d = tmp_path_factory.mktemp("abi")
    (d / "layout.c").write_text(SOURCE)
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(d / "layout.c"), "-o", str(d / "layout")], check=True)
    out = subprocess.run([str(d / "layout")], check=True, capture_output=True, text=True).stdout
    return {k: (int(a), int(b)) for k, a, b in (line.split() for line in out.splitlines())}


def test_structs(laid_out):
    from paper_2602_01665_amd import binding as B
    for s in (B.TabxHeads, B.TabxAxis):
        assert C.sizeof(s) == laid_out[f"sizeof({s.__name__})"][0]
        for name, _ in s._fields_:
            field = getattr(s, name)
            assert (field.offset, field.size) == laid_out[f"{s.__name__}.{name}"], name
        assert len(s._fields_) == sum(k.startswith(s.__name__ + ".") for k in laid_out)
    assert laid_out["sizeof(TabxHeads)"][0] == 40 and laid_out["sizeof(TabxAxis)"][0] == 24


def test_constants(laid_out):
    import torch

    from paper_2602_01665_amd import binding as B
    assert [laid_out["TABX_" + n][0] for n in ("F32", "BF16", "F16", "E4M3", "I32")] == [0, 1, 2, 3, 4]
    assert B._NARROW[torch.float8_e4m3fn] == 3 and B._INT == 4 and torch.float8_e4m3fn not in B.TYPES
    assert laid_out["TABX_ROTARY_MAX_WIDTH"][0] == 512 and laid_out["TABX_ROTARY_MAX_AXES"][0] == 4
    most, heads = laid_out["TABX_ATTENTION_MAX_WIDTH"][0], laid_out["TABX_ATTENTION_MAX_HEADS"][0]
    assert B.tabx_linear_attention_workspace(1 << 20, 1, 1, most, most) > 0
    for bad in ((4, 4, 1, most + 1, 4), (4, 4, 1, 4, most + 1), (4, 4, heads + 1, 4, 4)):
        with pytest.raises(B.TabxError):
            B.tabx_linear_attention_workspace(*bad)
