"""Linear attention of values so large that a product of matrices would leave 32 bits, or a part of 16 bits would not be
finite, though the recurrence's sums stay in range: what comes out is what the recurrence gives."""
import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
MOST = {F32: 3.4e38, BF16: 3.3e38, F16: 65504.0}


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def queries(d, dtype):
    """One of them nearly the largest there is; memory and gradients are small."""
    for n in ("v", "grad_out", "state"):
        d[n] *= 1e-6
    d["q"][20, 0, 0, 2] = MOST[dtype]
    d["grad_state"] *= 1e-3


def values(d, dtype):
    for n in ("q", "grad_out", "k"):
        d[n] *= 1e-4
    d["v"][21, 0, 0, 1], d["k"][25, 0, 0, 2] = -MOST[dtype] / 4, MOST[dtype] / 1e10
    d["v"][25, 0, 0] *= 1e-3


def values_alone(d, dtype):
    """v grad_out is beyond 32 bits where v alone is large, in ticks of their own."""
    d["k"][:, 0, 0] *= 1e-9
    d["q"][:, 0, 0] *= 1e-9
    d["state"] *= 1e-9
    d["grad_state"] *= 1e-9
    d["grad_out"][:, 0, 0] *= 1e8
    d["v"][5, 0, 0] *= 1e31 if dtype is F32 else 1e30
    d["k"][5, 0, 0] *= 1e-30
    d["log_decay"][0] = 0.0


def gradients(d, dtype):
    for n in ("q", "v", "k", "state"):
        d[n] *= 1e-4
    d["grad_out"][30, 0, 0, 3] = MOST[dtype]


def scores(d, dtype):
    """q k is beyond 32 bits, k v and q (k v) are not."""
    d["k"][5, 0, 0] *= 1e20
    d["v"][5, 0, 0] *= 1e-30
    d["q"][9, 0, 0] *= 1e20
    d["grad_out"][9, 0, 0] *= 1e-30


def scores_of_values(d, dtype):
    d["v"][5, 0, 0] *= 1e20
    d["k"][5, 0, 0] *= 1e-30
    d["grad_out"][9, 0, 0] *= 1e20
    d["q"][9, 0, 0] *= 1e-30


def state(d, dtype):
    """One element nearly the largest there is, which nothing reads; and one of the gradient's."""
    d["state"][0, 0, 3, 1] = 3.4e38
    d["grad_state"][0, 0, 2, 0] = -3.4e38
    d["q"][:, 0, 0, 3] = 0.0
    d["grad_out"][:, 0, 0, 1] = 0.0
    d["k"][:, 0, 0, 2] = 0.0
    d["v"][:, 0, 0, 0] = 0.0


def faded(d, dtype):
    """A state that is out of its queries' range before it has faded, and in it afterwards."""
    d["log_decay"] = torch.full_like(d["log_decay"], -5.0)
    d["state"][0, 0] *= 1e30
    d["grad_state"][0, 0] *= 1e30
    for n in ("q", "k", "v", "grad_out"):
        d[n][:, 0, 0] *= 1e-9
    d["q"][3, 0, 0] *= 1e17
    d["grad_out"][3, 0, 0] *= 1e17
    d["k"][-4, 0, 0] *= 1e17
    d["v"][-4, 0, 0] *= 1e17


def scale(d, dtype):
    d["scale"] = 1e30
    for n in ("q", "k"):
        d[n] *= 1e5
    for n in ("v", "grad_out"):
        d[n] *= 1e-33
    d["state"] *= 1e-28


def cancelled(d, dtype):
    """Two ticks of which the second takes back the first: each alone would be beyond 32 bits for a later query."""
    d["log_decay"][0] = 0.0
    d["fresh"][:] = 0
    d["k"][5, 0, 0], d["v"][5, 0, 0] = d["k"][5, 0, 0] * 1e14, d["v"][5, 0, 0] * 1e14
    d["k"][6, 0, 0], d["v"][6, 0, 0] = d["k"][5, 0, 0], -d["v"][5, 0, 0]
    for n in ("q", "grad_out"):
        d[n][:7, 0, 0] *= 1e-14
    d["q"][8, 0, 0] *= 1e13
    for n in ("grad_out", "grad_state"):
        (d[n] if n == "grad_state" else d[n][:, 0, 0]).mul_(1e-14)


PLANTS = [queries, values, values_alone, gradients, scores, scores_of_values, state, faded, scale, cancelled]
# (f16 ends where all of this begins: its states only, whatever they hold)
CASES = [(p, t) for p in PLANTS for t in (F32, BF16)] + [(state, F16)]


def make(T, R, H, K, V, dtype, plant=None):
    g = torch.Generator().manual_seed(T + K)
    d = {n: torch.randn(T, R, H, w, generator=g) for n, w in (("q", K), ("k", K), ("v", V), ("grad_out", V))}
    d["fresh"] = (torch.rand(T, R, generator=g) < 0.02).to(torch.uint8)
    d["fresh"][:32, 0] = 0
    d["state"], d["grad_state"] = (torch.randn(R, H, K, V, generator=g) for _ in range(2))
    d["log_decay"], d["scale"] = M.decays(H) / 4, K ** -0.5
    if plant is not None:
        plant(d, dtype)
    return {n: x.to(dtype) if n in ("q", "k", "v", "grad_out") else x for n, x in d.items()}


def expected(d):
    c = (d["q"], d["k"], d["v"], d["log_decay"], d["scale"], d["fresh"], d["state"])
    want = dict(M.attention(*c), **M.attention_grad(*c, d["grad_out"], d["grad_state"]))
    # out = scale * (q S) and grad_q = scale * (S grad_out) multiply by the scale last.  Of the sum's K or V terms each is the
    # product of two 32-bit numbers; one below 2^-126 may be rounded to zero, that is off by up to 2^-126, and the partial sums
    # after it too, 2 * 128 * 2^-126 at most together, which the scale multiplies.  (For a scale of up to one that is what the
    # bounds hold already; for one of 1e30 and elements of 1e-33 it is all of grad_q.)
    lost = abs(d["scale"]) * 2 * 128 * 2.0 ** -126
    return {n: (value, bound + lost if n in ("out", "grad_q") else bound) for n, (value, bound) in want.items()}


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


def steps(B, d):
    up = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in d.items()}
    after, out = up["state"].clone(), torch.empty_like(up["v"])
    for t in range(len(out)):
        B.tabx_linear_attention_step(up["q"][t], up["k"][t], up["v"][t], up["log_decay"], up["scale"], after, out[t], up["fresh"][t])
    return {"out": out, "state_out": after}


@pytest.mark.parametrize("plant,dtype", CASES, ids=lambda x: getattr(x, "__name__", str(x)))
@pytest.mark.parametrize("shape", [(50, 2, 2, 16, 16), (70, 1, 2, 64, 48), (40, 2, 1, 96, 80), (140, 1, 2, 128, 100)], ids=str)
def test_what_32_bits_hold_they_hold(B, shape, plant, dtype):
    d = make(*shape, dtype, plant)
    want = expected(d)
    for n, (value, _) in want.items():
        assert float(value.abs().max()) < (3.4e38 if "state" in n else MOST[dtype]), n
    for n, x in run(B, d).items():
        M.near(x, *want[n], n)
    for n, x in steps(B, d).items():
        M.near(x, *want[n], ("step", n))


@pytest.mark.parametrize("plant", PLANTS, ids=lambda p: p.__name__)
@pytest.mark.parametrize("K,V,dtype", [(64, 64, BF16), (128, 128, BF16), (40, 40, F32)], ids=str)
def test_other_rows_are_as_they_were(B, plant, K, V, dtype):
    """The ticks of many rows, whole (no segments): the rows beside a planted one bit for bit; its copies each the same."""
    T, R = 200, 1100
    assert B.tabx_linear_attention_workspace(T, R, 1, K, V) == 0
    base = make(T, 2, 1, K, V, dtype, plant)
    want = expected(base)
    some = torch.zeros(R, dtype=torch.long)
    some[1::2] = 1

    def many(rows):
        return run(B, {n: x[rows] if "state" in n else x[:, rows] if isinstance(x, torch.Tensor) and n != "log_decay" else x
                       for n, x in base.items()})

    whole, plain = many(some), many(torch.ones(R, dtype=torch.long))
    for n, x in whole.items():
        k = 0 if "state" in n else 1
        a, b = x.select(k, 0), x.select(k, 1)
        assert torch.equal(x.index_select(k, torch.arange(0, R, 2, device="cuda")), a.unsqueeze(k).expand_as(x.index_select(k, torch.arange(0, R, 2, device="cuda")))), n
        assert torch.equal(b, plain[n].select(k, 1)), n
        M.near(torch.stack((a, b), k), *want[n], n)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("T,K,V", [(40, 128, 128), (130, 64, 64), (130, 96, 96), (2100, 16, 16)])
def test_products_of_matrices_up_to_their_limits(B, T, K, V, dtype):
    """All elements just below 2^30, a scale of 2^16, a state of nearly 2^70 that grows beyond it: the largest sums there
    are before a chunk goes tick by tick, all of one sign."""
    d = make(T, 1, 2, K, V, dtype)
    for n in ("q", "k", "v", "grad_out"):
        d[n] = torch.full_like(d[n], 2.0 ** 30 - 2.0 ** 22)
    d["state"], d["grad_state"] = torch.full_like(d["state"], 2.0 ** 70 - 2.0 ** 60), torch.full_like(d["grad_state"], 2.0 ** 70 - 2.0 ** 60)
    d["fresh"][:], d["log_decay"], d["scale"] = 0, torch.tensor([0.0, -1e-4]), 2.0 ** 16
    want = expected(d)
    for n, (value, _) in want.items():
        assert 2.0 ** 60 < float(value.abs().max()) < 2.0 ** 127, n
    for n, x in run(B, d).items():
        M.near(x, *want[n], n)


@pytest.mark.parametrize("grows", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_rows_of_more_chunks_than_a_state_is_trusted_for(B, dtype, grows):
    """More than 64 chunks of one workgroup: a state that stays small, and one that has grown past 2^70 by then."""
    T, R, K, V = 2200, 1100, 8, 8
    assert B.tabx_linear_attention_workspace(T, R, 1, K, V) == 0
    d = make(T, 1, 1, K, V, dtype)
    d["log_decay"] = torch.zeros(1)
    if grows:
        for n in ("q", "k", "v", "grad_out"):
            d[n] = torch.full_like(d[n], 2.0 ** 30 - 2.0 ** 22)
        d["fresh"][:] = 0
    want = expected(d)
    assert (float(want["state_out"][0].abs().max()) > 2.0 ** 70) == grows
    got = run(B, {n: x.expand(R, *x.shape[1:]).contiguous() if "state" in n else x.expand(T, R, *x.shape[2:]).contiguous()
                  if isinstance(x, torch.Tensor) and n != "log_decay" else x for n, x in d.items()})
    for n, x in got.items():
        one = x.narrow(0 if "state" in n else 1, 0, 1)
        assert torch.equal(x, one.expand_as(x)), n
        M.near(one, *want[n], n)
