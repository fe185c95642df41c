"""Linear attention as an update calls it: so many rows that every workgroup goes through all of a row's chunks, in every
width's form and type; a few ticks of them; and calls of more heads than a launch has workgroups."""
import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def make(T, R, H, K, V, dtype, ends):
    g = torch.Generator().manual_seed(T + K + V)
    d = {n: (torch.randn(T, R, H, w, generator=g) * w ** -0.25).to(dtype) for n, w in (("q", K), ("k", K))}
    d["v"], d["grad_out"] = (torch.randn(T, R, H, V, generator=g).to(dtype) for _ in range(2))
    d["fresh"] = (torch.rand(T, R, generator=g) < ends).to(torch.uint8)
    d["state"], d["grad_state"] = (torch.randn(R, H, K, V, generator=g) for _ in range(2))
    d["log_decay"], d["scale"] = M.decays(H), K ** -0.5
    return d


def expected(d):
    """f16 results are held to the bounds of 32 bits, rounded to f16; bf16 ones to those of their own type's."""
    x = {n: d[n].float() if d["q"].dtype is F16 else d[n] for n in ("q", "k", "v", "grad_out")}
    c = (x["q"], x["k"], x["v"], d["log_decay"], d["scale"], d["fresh"], d["state"])
    want = dict(M.attention(*c), **M.attention_grad(*c, x["grad_out"], d["grad_state"]))
    if d["q"].dtype is F16:
        want = {n: (v, b if "state" in n else M.rounded(b, v, F16)) for n, (v, b) in want.items()}
    return want


def copies(d, n):
    """Each row n times, side by side, on the GPU."""
    of = {}
    for name, x in d.items():
        if isinstance(x, torch.Tensor) and name != "log_decay":
            x = x.cuda().repeat_interleave(n, 0 if "state" in name else 1)
        of[name] = x.cuda() if isinstance(x, torch.Tensor) else x
    return of


def run(B, up):
    T, R, H, K = up["q"].shape
    V, dtype = up["v"].shape[-1], up["q"].dtype
    need = B.tabx_linear_attention_workspace(T, R, H, K, V)
    assert need == 0, "cut into segments"
    got = {n: torch.full((T, R, H, w), 7.0, dtype=dtype, device="cuda") for n, w in (("out", V), ("grad_q", K), ("grad_k", K), ("grad_v", V))}
    got["state_out"], got["grad_state_in"] = (torch.full((R, H, K, V), 7.0, device="cuda") for _ in range(2))
    c = (up["q"], up["k"], up["v"], up["log_decay"], up["scale"])
    B.tabx_linear_attention(*c, got["out"], up["fresh"], up["state"], got["state_out"])
    B.tabx_linear_attention_backward(*c, up["grad_out"], got["grad_q"], got["grad_k"], got["grad_v"], up["fresh"], up["state"],
                                     up["grad_state"], got["grad_state_in"])
    return got


def check(B, d, n):
    want = expected(d)
    for name, x in run(B, copies(d, n)).items():
        k = 0 if "state" in name else 1
        x = x.unflatten(k, (-1, n))
        one = x.narrow(k + 1, 0, 1)
        assert torch.equal(x, one.expand_as(x)), name                  # the copies are the same bits
        M.near(one.squeeze(k + 1), *want[name], name)


WIDTHS = [(32, 32), (20, 27), (64, 64), (40, 64), (33, 50), (96, 96), (70, 96), (128, 128), (97, 128), (128, 30)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("K,V", WIDTHS)
def test_rows_of_many_chunks(B, K, V, dtype):
    check(B, make(203, 3, 2, K, V, dtype, 0.015), 350)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("K,V", [(32, 32), (64, 64), (50, 64), (96, 96), (96, 65), (128, 128), (120, 128)])
def test_rows_of_few_ticks(B, K, V, dtype):
    for T in (1, 2, 8, 31, 32):
        check(B, make(T, 5, 2, K, V, dtype, 0.1), 2)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("K,V", [(32, 32), (64, 48), (96, 96), (128, 128)])
def test_steps_against_ticks_at_once(B, K, V, dtype):
    """A rollout's and an update's results of the same ticks, whose values nearly take each other back."""
    T, R, H = 70, 4, 2
    d = make(T, R, H, K, V, dtype, 0.05)
    for x, sign in (("k", 1.0), ("v", -1.0)):
        d[x][1::2] = (d[x][0::2].float() * sign * (1.0 + 2.0 ** -6 * torch.rand(d[x][0::2].shape, generator=torch.Generator().manual_seed(1)))).to(dtype)
    want = expected(d)
    up = copies(d, 1)
    steps, after = torch.empty_like(up["v"]), up["state"].clone()
    for t in range(T):
        B.tabx_linear_attention_step(up["q"][t], up["k"][t], up["v"][t], up["log_decay"], up["scale"], after, steps[t], up["fresh"][t])
    out, last = torch.empty_like(steps), torch.empty_like(after)
    ws = torch.empty(B.tabx_linear_attention_workspace(T, R, H, K, V), dtype=torch.uint8, device="cuda")
    B.tabx_linear_attention(up["q"], up["k"], up["v"], up["log_decay"], up["scale"], out, up["fresh"], up["state"], last, ws)
    for name, a, b in (("out", steps, out), ("state_out", after, last)):
        M.near(a, *want[name], ("steps", name))
        M.near(b, *want[name], ("at once", name))
        M.near(b, M.f64(a), 2 * want[name][1], name)


@pytest.mark.parametrize("dtype,works", [(BF16, 2 ** 20 + 1025), (F32, 2 ** 19 + 77)], ids=str)
def test_gradients_of_more_heads_than_a_launch_has_workgroups(B, dtype, works):
    """(in f32, three workgroups to a head)"""
    T, H, K, V = 2, 1, 4, 4
    g = torch.Generator("cuda").manual_seed(works)
    up = {n: torch.randn(T, works, H, w, generator=g, device="cuda").to(dtype) for n, w in (("q", K), ("k", K), ("v", V), ("grad_out", V))}
    up["fresh"] = (torch.rand(T, works, generator=g, device="cuda") < 0.3).to(torch.uint8)
    up["state"], up["grad_state"] = (torch.randn(works, H, K, V, generator=g, device="cuda") for _ in range(2))
    up["log_decay"], up["scale"] = M.decays(H).cuda(), 0.5
    whole = run(B, up)
    for at in (0, 2 ** 20 // 3 - 3, 2 ** 19 - 3, works - 6):
        few = {n: (x[at:at + 6] if "state" in n else x[:, at:at + 6].contiguous()) if isinstance(x, torch.Tensor) and n != "log_decay" else x
               for n, x in up.items()}
        for n, x in run(B, few).items():
            assert torch.equal(whole[n].narrow(0 if "state" in n else 1, at, 6), x), (n, at)
    few = {n: x.cpu() if isinstance(x, torch.Tensor) else x for n, x in few.items()}
    for n, (value, bound) in expected(few).items():
        M.near(whole[n].narrow(0 if "state" in n else 1, works - 6, 6), value, bound, n)


@pytest.mark.parametrize("K,V,dtype,works", [(1, 4, BF16, 2 ** 25 + 1025), (17, 4, F32, 2 ** 22 + 333), (3, 1, F16, 2 ** 22 + 333)], ids=str)
def test_steps_of_more_heads_than_a_launch_has_workgroups(B, K, V, dtype, works):
    """Lanes, wavefronts and odd values that take a second turn: out and state are those of the same rows a few at a time."""
    g = torch.Generator("cuda").manual_seed(works)
    q, k, v = (torch.randn(works, 1, w, generator=g, device="cuda").to(dtype) for w in (K, K, V))
    fresh = (torch.rand(works, generator=g, device="cuda") < 0.3).to(torch.uint8)
    state, decay = torch.randn(works, 1, K, V, generator=g, device="cuda"), M.decays(1).cuda()
    places = [slice(at, at + 5) for at in (0, works // 2, 2 ** 20 - 2, 2 ** 22 - 2, works - 5)]
    before = [state[s].clone() for s in places]
    out = torch.full_like(v, 7.0)
    B.tabx_linear_attention_step(q, k, v, decay, 0.5, state, out, fresh)
    for s, own in zip(places, before):
        want = M.attention(q[s].cpu()[None], k[s].cpu()[None], v[s].cpu()[None], M.decays(1), 0.5, fresh[s].cpu()[None], own.cpu())
        one = torch.full_like(v[s], 7.0)
        B.tabx_linear_attention_step(q[s], k[s], v[s], decay, 0.5, own, one, fresh[s])
        assert torch.equal(out[s], one) and torch.equal(state[s], own), s
        M.near(one[None], *want["out"], s)
        M.near(own, *want["state_out"], s)
