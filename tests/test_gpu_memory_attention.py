"""Linear attention with a decay for each head, one tick and many, and its gradients, against the recurrence
in 64 bits."""
import math

import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def generator(seed):
    return torch.Generator().manual_seed(seed)


def make(seed, T, R, H, K, V, dtype, units=1, ends=0.1, joined=False):
    """Inputs on the host: q, k, v, grad_out, fresh [T, R / units], state, grad_state, log_decay."""
    g = generator(seed)
    q, k = (torch.randn(T, R, H, K, generator=g) * K ** -0.25 for _ in range(2))
    v, go = (torch.randn(T, R, H, V, generator=g) for _ in range(2))
    d = {"q": q, "k": k, "v": v, "grad_out": go}
    d = {n: x.to(dtype) for n, x in d.items()}
    d["fresh"] = (torch.rand(T, R // units, generator=g) < ends).to(torch.uint8)
    d["state"], d["grad_state"] = (torch.randn(R, H, K, V, generator=g) for _ in range(2))
    d["log_decay"], d["scale"] = M.decays(H), K ** -0.5
    return d


def on_gpu(d):
    return {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in d.items()}


def workspace(B, T, R, H, K, V, dev="cuda"):
    return torch.empty(B.tabx_linear_attention_workspace(T, R, H, K, V), dtype=torch.uint8, device=dev).fill_(255)


def forward(B, d, fresh=True, state=True, controlled=None, **kw):
    T, R, H, K = d["q"].shape
    V = d["v"].shape[-1]
    out = torch.full((T, R, H, V), 7.0, dtype=d["q"].dtype, device="cuda")
    after = torch.full((R, H, K, V), 7.0, device="cuda")
    B.tabx_linear_attention(d["q"], d["k"], d["v"], d["log_decay"], d["scale"], out, d["fresh"] if fresh else None,
                            d["state"] if state else None, after, workspace(B, T, R, H, K, V), controlled, **kw)
    return {"out": out, "state_out": after}


def backward(B, d, fresh=True, state=True, controlled=None):
    T, R, H, K = d["q"].shape
    V = d["v"].shape[-1]
    gq, gk = (torch.full((T, R, H, K), 7.0, dtype=d["q"].dtype, device="cuda") for _ in range(2))
    gv = torch.full((T, R, H, V), 7.0, dtype=d["q"].dtype, device="cuda")
    gs = torch.full((R, H, K, V), 7.0, device="cuda")
    B.tabx_linear_attention_backward(d["q"], d["k"], d["v"], d["log_decay"], d["scale"], d["grad_out"], gq, gk, gv,
                                     d["fresh"] if fresh else None, d["state"] if state else None,
                                     d["grad_state"] if state else None, gs, workspace(B, T, R, H, K, V), controlled)
    return {"grad_q": gq, "grad_k": gk, "grad_v": gv, "grad_state_in": gs}


def expected(d, fresh=True, state=True):
    return M.attention(d["q"], d["k"], d["v"], d["log_decay"], d["scale"], d["fresh"] if fresh else None,
                       d["state"] if state else None)


def expected_grad(d, fresh=True, state=True):
    return M.attention_grad(d["q"], d["k"], d["v"], d["log_decay"], d["scale"], d["fresh"] if fresh else None,
                            d["state"] if state else None, d["grad_out"], d["grad_state"] if state else None)


def compare(got, want, what):
    for n, x in got.items():
        M.near(x, want[n][0], want[n][1], f"{what}: {n}")


# ticks around the chunks' ends; widths of every form, odd ones, keys and values of different ones
SHAPES = [(1, 3, 2, 16, 16), (2, 2, 3, 8, 24), (31, 2, 2, 32, 32), (32, 2, 1, 5, 3), (33, 2, 2, 16, 16), (64, 1, 2, 64, 64),
          (65, 3, 1, 1, 1), (63, 2, 2, 17, 33), (97, 1, 2, 128, 128), (128, 1, 1, 40, 128), (40, 2, 1, 127, 65),
          (129, 1, 3, 48, 80), (300, 1, 1, 20, 20)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_many_ticks(B, shape, dtype):
    d = make(1, *shape, dtype)
    for fresh, state in ((True, True), (False, False)):
        compare(forward(B, on_gpu(d), fresh, state), expected(d, fresh, state), (shape, dtype, fresh))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients(B, shape, dtype):
    d = make(2, *shape, dtype)
    for fresh, state in ((True, True), (False, False)):
        compare(backward(B, on_gpu(d), fresh, state), expected_grad(d, fresh, state), (shape, dtype, fresh))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(1, 6, 2, 16, 16), (1, 5, 3, 8, 24), (1, 4, 1, 32, 32), (1, 7, 2, 1, 1), (1, 3, 2, 17, 33),
                                   (1, 2, 2, 64, 64), (1, 2, 1, 128, 128), (1, 3, 1, 127, 65), (1, 4, 4, 4, 100)], ids=str)
def test_one_tick(B, shape, dtype):
    d = make(3, *shape, dtype, ends=0.4)
    g = on_gpu(d)
    want = expected(d)
    out, state = torch.full_like(g["v"][0], 7.0), g["state"].clone()
    B.tabx_linear_attention_step(g["q"][0], g["k"][0], g["v"][0], g["log_decay"], d["scale"], state, out, g["fresh"][0])
    M.near(out, want["out"][0][0], want["out"][1][0], (shape, dtype))
    M.near(state, *want["state_out"], (shape, dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_few_rows_of_many_ticks_are_cut_into_segments(B, dtype):
    """An episode that ends in a segment, one that spans several, none at all."""
    for seed, (T, R, H, K, V), ends in ((4, (1000, 1, 2, 24, 16), 0.002), (5, (700, 2, 1, 64, 64), 0.0), (6, (513, 1, 1, 100, 128), 0.05)):
        d = make(seed, T, R, H, K, V, dtype, ends=ends)
        assert B.tabx_linear_attention_workspace(T, R, H, K, V) > 0
        compare(forward(B, on_gpu(d)), expected(d), (T, dtype))
        compare(backward(B, on_gpu(d)), expected_grad(d), (T, dtype))


def test_ticks_one_by_one_are_ticks_at_once(B):
    """A rollout's steps against one call over its ticks: the same sums in another order."""
    T, R, H, K, V = 70, 12, 2, 32, 24
    d = make(7, T, R, H, K, V, torch.float32, units=3)
    g = on_gpu(d)
    want = expected(d)
    state, outs = g["state"].clone(), []
    for t in range(T):
        out = torch.empty(R, H, V, device="cuda")
        B.tabx_linear_attention_step(g["q"][t], g["k"][t], g["v"][t], g["log_decay"], d["scale"], state, out, g["fresh"][t])
        outs.append(out)
    M.near(torch.stack(outs), *want["out"], "steps")
    M.near(state, *want["state_out"], "steps")
    got = forward(B, g)
    compare(got, want, "at once")
    M.near(got["out"], M.f64(torch.stack(outs)), 2 * want["out"][1], "one against the other")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_rows_left_out(B, dtype):
    T, R, H, K, V = 45, 10, 2, 16, 40
    d = make(8, T, R, H, K, V, dtype, units=5)
    controlled = torch.tensor([1, 0, 1, 1, 0] * 2, dtype=torch.uint8)
    out_of = controlled == 0
    for n in ("q", "k", "v", "grad_out"):
        d[n][:, out_of] = NAN
    for n in ("state", "grad_state"):
        d[n][out_of] = NAN
    g = on_gpu(d)
    clean = {n: torch.nan_to_num(x) if isinstance(x, torch.Tensor) and x.is_floating_point() else x for n, x in d.items()}
    on = controlled != 0

    def check(got, want, axis, left):
        for n, x in got.items():
            x, (value, bound) = x.cpu(), want[n]
            k = 0 if "state" in n else axis
            M.near(x.index_select(k, on.nonzero()[:, 0]), value.index_select(k, on.nonzero()[:, 0]),
                   bound.index_select(k, on.nonzero()[:, 0]), n)
            assert (x.index_select(k, out_of.nonzero()[:, 0]) == left).all(), n

    check(forward(B, g, controlled=controlled.cuda()), expected(clean), 1, 7.0)
    check(backward(B, g, controlled=controlled.cuda()), expected_grad(clean), 1, 0.0)
    one, state, out = {n: x[:1] for n, x in clean.items() if n in ("q", "k", "v", "fresh")}, g["state"].clone(), torch.full_like(g["v"][0], 7.0)
    B.tabx_linear_attention_step(g["q"][0], g["k"][0], g["v"][0], g["log_decay"], d["scale"], state, out, g["fresh"][0], controlled.cuda())
    want = M.attention(one["q"], one["k"], one["v"], d["log_decay"], d["scale"], one["fresh"], clean["state"])
    M.near(out.cpu()[on], want["out"][0][0][on], want["out"][1][0][on], "step")
    M.near(state.cpu()[on], want["state_out"][0][on], want["state_out"][1][on], "step")
    assert (out.cpu()[out_of] == 7.0).all() and torch.isnan(state.cpu()[out_of]).all()


@pytest.mark.parametrize("order", ["projection", "rows first", "shared head"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_strides(B, order, dtype):
    """Columns of one projection's output at odd places, rows before ticks, one key for all heads."""
    T, R, H, K, V = 37, 4, 3, 10, 18
    d = make(9, T, R, H, K, V, dtype, units=2)
    g = on_gpu(d)
    if order == "projection":
        wide = torch.full((T, R, 1 + H * (2 * K + V) + 2), NAN, dtype=dtype, device="cuda")
        at = 1
        for n, w in (("q", K), ("k", K), ("v", V)):
            view = wide[..., at:at + H * w].unflatten(-1, (H, w))
            view.copy_(g[n])
            g[n] = view
            at += H * w
    elif order == "rows first":
        for n in ("q", "k", "v", "grad_out"):
            x = torch.empty((R, H, T, g[n].shape[-1] + 3), dtype=dtype, device="cuda").permute(2, 0, 1, 3)[..., :-3]
            x.copy_(g[n])
            g[n] = x
    else:
        d["k"] = d["k"][:, :, :1].expand(T, R, H, K)
        g["k"] = g["k"][:, :, :1].expand(T, R, H, K)
    compare(forward(B, g), expected(d), order)
    compare(backward(B, g), expected_grad(d), order)
    # outputs that are columns of a wider array, whose others stay
    wide = torch.full((T, R, H * V + 5), 7.0, dtype=dtype, device="cuda")
    out = wide[..., 2:2 + H * V].unflatten(-1, (H, V))
    B.tabx_linear_attention(g["q"], g["k"], g["v"], g["log_decay"], d["scale"], out, g["fresh"], g["state"], None,
                            workspace(B, T, R, H, K, V))
    M.near(out, *expected(d)["out"], order)
    assert (wide[..., :2] == 7.0).all() and (wide[..., 2 + H * V:] == 7.0).all()


def test_state_in_place_and_on_its_own(B):
    T, R, H, K, V = 50, 3, 2, 16, 16
    d = make(10, T, R, H, K, V, torch.float32)
    g = on_gpu(d)
    want, want_grad = expected(d), expected_grad(d)
    state, out = g["state"].clone(), torch.empty_like(g["v"])
    B.tabx_linear_attention(g["q"], g["k"], g["v"], g["log_decay"], d["scale"], out, g["fresh"], state, state)
    M.near(state, *want["state_out"], "in place")
    M.near(out, *want["out"], "in place")
    for T2 in (50, 400):                                   # (whole, and in segments)
        d2 = make(11, T2, R, H, K, V, torch.float32, ends=0.01)
        g2, ws = on_gpu(d2), workspace(B, T2, R, H, K, V)
        gs, gv = g2["grad_state"].clone(), torch.empty_like(g2["v"])
        B.tabx_linear_attention_backward(g2["q"], g2["k"], g2["v"], g2["log_decay"], d2["scale"], g2["grad_out"], None, None, gv,
                                         g2["fresh"], g2["state"], gs, gs, ws)
        w2 = expected_grad(d2)
        M.near(gs, *w2["grad_state_in"], "in place")
        M.near(gv, *w2["grad_v"], "in place")
        for n in ("grad_q", "grad_k", "grad_v", "grad_state_in"):     # each alone
            one = {m: None for m in ("grad_q", "grad_k", "grad_v", "grad_state_in")}
            one[n] = torch.full(w2[n][0].shape, 7.0, device="cuda")
            B.tabx_linear_attention_backward(g2["q"], g2["k"], g2["v"], g2["log_decay"], d2["scale"], g2["grad_out"], one["grad_q"],
                                             one["grad_k"], one["grad_v"], g2["fresh"], g2["state"], g2["grad_state"],
                                             one["grad_state_in"], ws)
            M.near(one[n], *w2[n], n)
    assert want_grad


@pytest.mark.parametrize("K,V", [(20, 33), (96, 70)])
def test_state_gradient_in_place_of_many_heads(B, K, V):
    """More heads than the machine holds at a time, of one tick: each gradient reads what it is given, whoever is first."""
    T, R, H = 1, 1501, 3
    g = on_gpu(make(22, T, R, H, K, V, torch.float32))
    got = []
    for in_place in (False, True):
        given = g["grad_state"].clone()
        after = given if in_place else torch.empty_like(given)
        grads = [torch.empty_like(g[n]) for n in ("q", "k", "v")]
        B.tabx_linear_attention_backward(g["q"], g["k"], g["v"], g["log_decay"], 0.25, g["grad_out"], *grads, g["fresh"], g["state"],
                                         given, after, workspace(B, T, R, H, K, V))
        got.append(grads + [after])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_no_ticks_and_no_rows(B):
    R, H, K, V = 3, 2, 5, 6
    d = on_gpu(make(12, 1, R, H, K, V, torch.float32))
    e = {n: d[n][:0] for n in ("q", "k", "v", "grad_out", "fresh")}
    after = torch.full_like(d["state"], 7.0)
    for given in (d["state"], None):
        B.tabx_linear_attention(e["q"], e["k"], e["v"], d["log_decay"], 1.0, e["v"].clone(), e["fresh"], given, after)
        assert torch.equal(after, torch.zeros_like(after) if given is None else given)
        B.tabx_linear_attention_backward(e["q"], e["k"], e["v"], d["log_decay"], 1.0, e["grad_out"], None, None, None, e["fresh"],
                                         None, given, after)
        assert torch.equal(after, torch.zeros_like(after) if given is None else given)
    none = {n: d[n][:, :0] for n in ("q", "k", "v")}
    B.tabx_linear_attention(none["q"], none["k"], none["v"], d["log_decay"], 1.0, none["v"].clone(), None, None, None)
    B.tabx_linear_attention_step(none["q"][0], none["k"][0], none["v"][0], d["log_decay"], 1.0, d["state"][:0], none["v"][0].clone())
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_decays_at_their_ends(B, dtype):
    """None (0, above 0, NaN), all at once (-infinity), and so strong that powers vanish."""
    T, R, K, V = 70, 2, 16, 16
    given = torch.tensor([0.0, 3.0, NAN, -INF, -30.0, -200.0, -1e-4, -1e-30])
    d = make(13, T, R, len(given), K, V, dtype, ends=0.03)
    d["log_decay"] = given
    compare(forward(B, on_gpu(d)), expected(d), dtype)
    compare(backward(B, on_gpu(d)), expected_grad(d), dtype)


def test_episodes_that_begin_everywhere_and_at_the_ends(B):
    T, R, H, K, V = 66, 1, 2, 16, 16
    for begins in (range(T), [0], [T - 1], [31], [32], [33], [0, 31, 32, 33, 63, 64, 65]):
        d = make(14, T, R, H, K, V, torch.float32, ends=0.0)
        d["fresh"][list(begins)] = 200
        compare(forward(B, on_gpu(d)), expected(d), begins)
        compare(backward(B, on_gpu(d)), expected_grad(d), begins)


@pytest.mark.parametrize("what", [NAN, INF, -INF])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("T", [66, 300])
def test_what_is_not_finite_stays_in_its_episode(B, dtype, what, T):
    """A tick's q, k or v, or a state, reaches later ticks of its episode, its own head and no others."""
    R, H, K, V = 2, 2, 16, 24
    for name, t in (("v", 5), ("v", 40), ("v", T - 1), ("k", 5), ("k", 40), ("q", 5), ("state", 0)):
        d = make(15, T, R, H, K, V, dtype, ends=0.0)
        d["fresh"][[9, 50]] = 1
        clean = expected(d)
        (d["state"][0, 1] if name == "state" else d[name][t, 0, 1])[..., 3] = what
        got = forward(B, on_gpu(d))
        out, after = M.f64(got["out"]), M.f64(got["state_out"])
        end = min([e for e in (9, 50, T) if e > t])
        reached = torch.zeros(T, R, H, dtype=torch.bool)
        reached[t:(t + 1 if name == "q" else end), 0, 1] = True
        value, bound = clean["out"]
        M.near(out[~reached], value[~reached], bound[~reached], (name, t))
        columns = [3] if name in ("v", "state") else range(V)
        assert not torch.isfinite(out[reached][:, columns]).any(), (name, t)
        if name in ("v", "state"):
            rest = [c for c in range(V) if c != 3]
            M.near(out[..., rest], value[..., rest], bound[..., rest], (name, t))
        survives = end == T and name != "q"
        assert torch.isfinite(after[0, 1]).all() != survives, (name, t)
        M.near(after[1], clean["state_out"][0][1], clean["state_out"][1][1], (name, t))
        M.near(after[0, 0], clean["state_out"][0][0, 0], clean["state_out"][1][0, 0], (name, t))


def test_the_largest_values_stay_in_their_episode(B):
    """Finite ones whose 16-bit part is not: what comes before them, and the next episode, is as it would be."""
    T, R, H, K, V = 50, 1, 1, 16, 16
    d = make(21, T, R, H, K, V, torch.float32, ends=0.0)
    d["fresh"][30] = 1
    clean = expected(d)
    most = torch.finfo(torch.float32).max
    d["v"][20, 0, 0, 5], d["k"][25, 0, 0, 2] = most, -most
    out = M.f64(forward(B, on_gpu(d))["out"])
    value, bound = clean["out"]
    for t in (slice(0, 20), slice(30, T)):
        M.near(out[t], value[t], bound[t], t)


def test_gradients_against_differences(B):
    """The 64-bit gradients of the reference are the slopes of its sums, and the call's are those."""
    T, R, H, K, V = 9, 2, 2, 4, 3
    d = make(16, T, R, H, K, V, torch.float32, ends=0.2)
    want = expected_grad(d)

    def total(e):
        x = {n: e[n].double() if e[n].dtype is torch.float32 and n != "log_decay" else e[n] for n in ("q", "k", "v", "state")}
        r = M.attention(x["q"], x["k"], x["v"], e["log_decay"], e["scale"], e["fresh"], x["state"])
        return float((r["out"][0] * d["grad_out"].double()).sum() + (r["state_out"][0] * d["grad_state"].double()).sum())

    M.STEP[torch.float64] = (2.0 ** -53, 0.0)
    try:
        g = generator(17)
        for name in ("q", "k", "v", "state"):
            along = torch.randn(d[name].shape, generator=g).double()
            slope = float((want["grad_state_in" if name == "state" else f"grad_{name}"][0] * along).sum())
            h = 2.0 ** -12
            up, down = (total(dict(d, **{name: d[name].double() + s * h * along})) for s in (1, -1))
            # the sums are at most quadratic in each input, so a central difference is off by roundings only
            assert abs((up - down) / (2 * h) - slope) < 1e-8 * (abs(slope) + 100.0), name
    finally:
        del M.STEP[torch.float64]
    compare(backward(B, on_gpu(d)), want, "call")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_equal_calls_give_equal_bits(B, dtype):
    for shape in ((100, 5, 2, 32, 48), (600, 1, 2, 64, 64)):
        g = on_gpu(make(18, *shape, dtype))
        a, b = dict(forward(B, g), **backward(B, g)), dict(forward(B, g), **backward(B, g))
        for n in a:
            assert torch.equal(a[n], b[n]), n


def test_many_rows_against_the_same_a_few_at_a_time(B):
    """More workgroups than a launch has, and offsets beyond 32 bits."""
    T, R, H, K, V = 2, 600001, 2, 4, 4
    g = torch.Generator("cuda").manual_seed(19)
    q, k, v = (torch.randn(T, R, H, K, generator=g, device="cuda") for _ in range(3))
    fresh = (torch.rand(T, R, generator=g, device="cuda") < 0.3).to(torch.uint8)
    state = torch.randn(R, H, K, V, generator=g, device="cuda")
    decay = M.decays(H).cuda()
    out, after = torch.empty_like(v), torch.empty_like(state)
    B.tabx_linear_attention(q, k, v, decay, 0.5, out, fresh, state, after)
    for at in (0, 300000, R - 5):
        s = slice(at, at + 5)
        o, a = torch.empty_like(v[:, s].contiguous()), torch.empty_like(state[s])
        B.tabx_linear_attention(q[:, s], k[:, s], v[:, s], decay, 0.5, o, fresh[:, s].contiguous(), state[s], a)
        assert torch.equal(out[:, s], o) and torch.equal(after[s], a)
    one = torch.empty_like(v[0])
    B.tabx_linear_attention_step(q[0], k[0], v[0], decay, 0.5, state, one, fresh[0])
    want = M.attention(q[:1, -5:].cpu(), k[:1, -5:].cpu(), v[:1, -5:].cpu(), M.decays(H), 0.5, fresh[:1, -5:].cpu(), None)
    assert torch.isfinite(one).all() and want


def test_offsets_beyond_32_bits(B):
    """Ticks that lie more than 2^32 elements apart, as columns of a very wide array."""
    T, R, H, K, V = 3, 2, 1, 8, 8
    d = make(20, T, R, H, K, V, torch.bfloat16)
    g = on_gpu(d)
    wide = torch.empty(T, 2 ** 31 + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    for n in ("q", "k", "v"):
        at = {"q": 2 ** 31, "k": 0, "v": 2 ** 30 + 1}[n]
        view = wide[:, at:at + R * H * K].unflatten(-1, (R, H, K))
        view.copy_(g[n])
        g[n] = view
    out = wide[:, 2 ** 31 + 4096:2 ** 31 + 4096 + R * H * V].unflatten(-1, (R, H, V))
    B.tabx_linear_attention(g["q"], g["k"], g["v"], g["log_decay"], d["scale"], out, g["fresh"], g["state"], None)
    M.near(out, *expected(d)["out"], "far")
