"""Linear attention and its gradients with a NaN or an infinity among the inputs: it reaches what the recurrences have it in,
and nothing else; not the other ticks of a chunk, not the next episode, not the one before, no other head and no other row."""
import math

import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INPUTS = ["q", "k", "v", "grad_out", "state", "grad_state"]


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def make(T, R, H, K, V, dtype):
    g = torch.Generator().manual_seed(T + K)
    d = {n: torch.randn(T, R, H, w, generator=g).to(dtype) for n, w in (("q", K), ("k", K), ("v", V), ("grad_out", V))}
    d["state"], d["grad_state"] = (torch.randn(R, H, K, V, generator=g) for _ in range(2))
    d["fresh"] = torch.zeros(T, R, dtype=torch.uint8)
    for t in {9, min(50, T - 1), T - 3}:           # row 0: episodes of less than a chunk, of several, of the last ticks
        d["fresh"][t, 0] = 1
    d["log_decay"], d["scale"] = M.decays(H), K ** -0.5
    return d


def expected(d):
    c = (d["q"], d["k"], d["v"], d["log_decay"], d["scale"], d["fresh"], d["state"])
    return dict(M.attention(*c), **M.attention_grad(*c, d["grad_out"], d["grad_state"]))


def run(B, d):
    up = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in d.items()}
    T, R, H, K = d["q"].shape
    V, dtype = d["v"].shape[-1], d["q"].dtype
    ws = torch.empty(B.tabx_linear_attention_workspace(T, R, H, K, V), dtype=torch.uint8, device="cuda")
    got = {n: torch.full((T, R, H, w), 7.0, dtype=dtype, device="cuda") for n, w in (("out", V), ("grad_q", K), ("grad_k", K), ("grad_v", V))}
    got["state_out"], got["grad_state_in"] = (torch.full((R, H, K, V), 7.0, device="cuda") for _ in range(2))
    c = (up["q"], up["k"], up["v"], up["log_decay"], up["scale"])
    B.tabx_linear_attention(*c, got["out"], up["fresh"], up["state"], got["state_out"], ws)
    B.tabx_linear_attention_backward(*c, up["grad_out"], got["grad_q"], got["grad_k"], got["grad_v"], up["fresh"], up["state"],
                                     up["grad_state"], got["grad_state_in"], ws)
    return got


def plant(d, name, t, what):
    d = dict(d, **{name: d[name].clone()})
    if "state" in name:
        d[name][0, 1, 2, 3] = what
    else:
        d[name][t, 0, 1, 3] = what
    return d


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("shape", [(70, 2, 2, 16, 24), (150, 1, 2, 64, 48), (60, 2, 2, 96, 80), (140, 1, 2, 128, 100)], ids=str)
def test_it_reaches_what_it_is_in(B, shape, dtype, what):
    d = make(*shape, dtype)
    T = shape[0]
    clean = run(B, d)
    for name in INPUTS:
        for t in (0,) if "state" in name else (0, 8, 9, 31, 40, 49, T - 4, T - 1):
            e = plant(d, name, t, what)
            got, want = run(B, e), expected(e)
            for n, x in got.items():
                M.near(x, *want[n], (name, t, n))
                h = 1 if "state" in n else 2                   # other heads and rows, bit for bit
                assert torch.equal(x.select(h, 0), clean[n].select(h, 0)), (name, t, n)
                assert torch.equal(x.narrow(h - 1, 1, x.shape[h - 1] - 1), clean[n].narrow(h - 1, 1, x.shape[h - 1] - 1)), (name, t, n)


@pytest.mark.parametrize("K,V,dtype", [(32, 32, BF16), (64, 64, BF16), (128, 128, BF16), (64, 64, F16), (40, 40, F32)], ids=str)
def test_it_does_in_whole_rows_of_many_chunks(B, K, V, dtype):
    """So many rows that no ticks are cut into segments: a workgroup goes through all of a row's chunks."""
    T, R = 150, 1100
    if K == 32:
        R = 2100
    assert B.tabx_linear_attention_workspace(T, R, 1, K, V) == 0
    base = make(T, 1, 2, K, V, dtype)
    base = {n: x[:, 1:] if n in ("state", "grad_state") else x[:, :, 1:] if n in ("q", "k", "v", "grad_out") else
            x[1:] if n == "log_decay" else x for n, x in base.items()}
    for name, t in (("q", 40), ("k", 40), ("v", 100), ("grad_out", 100), ("state", 0), ("grad_state", 0)):
        e = dict(base, **{name: base[name].clone()})
        (e[name][0, 0, 2] if "state" in name else e[name][t, 0, 0])[3] = math.nan
        got = run(B, {n: x.expand(R, *x.shape[1:]).contiguous() if "state" in n else x.expand(T, R, *x.shape[2:]).contiguous()
                      if isinstance(x, torch.Tensor) and n != "log_decay" else x for n, x in e.items()})
        want = expected(e)
        for n, x in got.items():
            k = 0 if "state" in n else 1
            one = x.narrow(k, 0, 1)
            assert torch.equal(torch.nan_to_num(x, 12345.0), torch.nan_to_num(one, 12345.0).expand_as(x)), (name, n)
            M.near(one, *want[n], (name, n))


@pytest.mark.parametrize("what", [math.nan, math.inf])
@pytest.mark.parametrize("K,V", [(16, 24), (16, 4), (33, 31), (7, 2)])
def test_steps_do_as_well(B, K, V, what):
    d = make(12, 2, 2, K, max(V, 4), F32)
    d = {n: x[..., :V].contiguous() if n in ("v", "grad_out", "state", "grad_state") else x for n, x in d.items()}
    for name, t in (("q", 3), ("k", 3), ("v", 3), ("state", 0)):
        e = dict(d, **{name: d[name].clone()})
        (e[name][0, 1, 2] if name == "state" else e[name][t, 0, 1])[1] = what
        want = M.attention(e["q"], e["k"], e["v"], e["log_decay"], e["scale"], e["fresh"], e["state"])
        up = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in e.items()}
        after, out = up["state"].clone(), torch.empty_like(up["v"])
        for i in range(len(out)):
            B.tabx_linear_attention_step(up["q"][i], up["k"][i], up["v"][i], up["log_decay"], up["scale"], after, out[i], up["fresh"][i])
        M.near(out, *want["out"], name)
        M.near(after, *want["state_out"], name)
