"""The learner's structs and constants as a C compiler lays them out, against the Python binding's
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
    VALUE(sizeof(TabxRows)); VALUE(sizeof(TabxSampling));
    FIELD(TabxRows, data); FIELD(TabxRows, stride); FIELD(TabxRows, type);
    FIELD(TabxSampling, temperature); FIELD(TabxSampling, top_k); FIELD(TabxSampling, top_p); FIELD(TabxSampling, min_p);
    VALUE(TABX_F32); VALUE(TABX_BF16); VALUE(TABX_F16); VALUE(TABX_NUM_ACTIONS);
    VALUE(TABX_NORM_MAX_WIDTH); VALUE(TABX_SAMPLE_MAX_LEVELS);
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
    for s in (B.TabxRows, B.TabxSampling):
        assert C.sizeof(s) == laid_out[f"sizeof({s.__name__})"][0]
        for name, _ in s._fields_:
            field = getattr(s, name)
            assert (field.offset, field.size) == laid_out[f"{s.__name__}.{name}"], name
        assert len(s._fields_) == sum(k.startswith(s.__name__ + ".") for k in laid_out)
    # what programs built against the header rely on
    assert laid_out["sizeof(TabxRows)"][0] == 24 and laid_out["sizeof(TabxSampling)"][0] == 24


def test_constants(laid_out):
    import torch

    from paper_2602_01665_amd import binding as B
    names = {torch.float32: "TABX_F32", torch.bfloat16: "TABX_BF16", torch.float16: "TABX_F16"}
    assert B.TYPES == {t: laid_out[n][0] for t, n in names.items()}
    assert laid_out["TABX_NUM_ACTIONS"][0] == B.tabx_num_actions() == 8
    assert laid_out["TABX_NORM_MAX_WIDTH"][0] == 8192 and laid_out["TABX_SAMPLE_MAX_LEVELS"][0] == 16384
    assert B.tabx_layer_norm_workspace(1, 8192) > 0
    with pytest.raises(B.TabxError):
        B.tabx_layer_norm_workspace(1, 8193)
