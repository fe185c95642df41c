"""Draws of actions and levels, and log-probabilities and their gradient, against 64-bit formulas
(needs an MI355X)."""
import numpy as np
import pytest
import torch

from tests import learner_reference as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda:0"
LOWEST = {F32: -3.4028234663852886e38, BF16: -3.3895313892515355e38, F16: -65504.0}
INF = float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def _say(*a):
    print("[gpu]", *a, flush=True)


def _logits(rng, rows, pad, dtype, kind, offset=0):
    v = rng.normal(size=(rows, 8)) * 2.0
    if kind == "coarse":                       # many equal scores
        v = np.round(v)
    elif kind == "equal":
        v[:] = 0.5
    elif kind == "wide":
        v *= 30.0
    elif kind == "odd":                        # what must not be chosen, in every form
        at = rng.random((rows, 8))
        v[at < 0.2] = -INF
        v[(at > 0.2) & (at < 0.3)] = np.nan
        v[(at > 0.3) & (at < 0.4)] = LOWEST[dtype]
        v[rng.random(rows) < 0.1] = -INF
        v[rng.random(rows) < 0.1] = LOWEST[dtype]
        v[rng.random(rows) < 0.05] = np.nan
        v[rng.random((rows, 8)) < 0.02] = INF
    whole = torch.full((offset + rows * (8 + pad),), 7.0, dtype=dtype, device=DEV)
    view = whole[offset:].view(rows, 8 + pad)[:, :8]
    view.copy_(torch.from_numpy(v))
    return whole, view


def _uniform(rng, rows):
    u = rng.random(rows).astype(np.float32)
    edge = np.array([0.0, 1.0, -1.0, np.nan, 1 - 2.0 ** -24, 0.5, 0.125, 2.0 ** -30, 1e-45, INF, 0.25, 0.375], np.float32)
    n = min(rows // 2, len(edge))
    u[:n] = edge[:n]
    return u


# (rows, pad, type, offset, kind, mask, controlled share, temperature, top_k, top_p, min_p)
DRAWS = [
    (1, 0, F32, 0, "normal", False, None, 1.0, 0, 1.0, 0.0), (96, 0, F32, 0, "normal", True, None, 1.0, 0, 1.0, 0.0),
    (255, 1, F32, 1, "odd", True, 0.5, 1.0, 0, 1.0, 0.0), (257, 0, BF16, 0, "odd", True, 0.5, 0.8, 5, 0.9, 0.02),
    (1000, 3, F16, 1, "odd", False, None, 1.3, 0, 0.7, 0.0), (3000, 1, BF16, 1, "coarse", True, 0.7, 0.5, 3, 1.0, 0.0),
    (3000, 0, F32, 0, "coarse", True, None, 1.0, 0, 0.5, 0.0), (999, 0, F32, 2, "equal", False, None, 2.0, 0, 0.5, 0.0),
    (999, 0, BF16, 0, "equal", True, None, 2.0, 3, 1.0, 1.0), (2000, 0, F32, 0, "wide", True, None, 1.0, 0, 0.999, 1e-6),
    (2000, 9, F16, 0, "coarse", True, 0.5, 0.0, 2, 0.5, 0.5), (700, 0, F32, 0, "odd", True, None, 0.0, 0, 1.0, 0.0),
    (2000, 0, F32, 0, "normal", True, None, 1.0, 1, 1.0, 0.0), (2000, 0, F32, 0, "normal", True, None, 1.0, 8, 1.0, 0.3),
    (2000, 0, F32, 0, "normal", False, None, 1.0, 100, 1e-6, 0.0), (2000, 0, BF16, 0, "coarse", False, None, 1.0, 4, 0.8, 0.1),
    (500, 0, F32, 0, "odd", True, 0.0, 1.0, 0, 1.0, 0.0), (600, 0, F32, 0, "normal", True, None, 1e-30, 0, 0.9, 0.0),
    (600, 0, F32, 0, "wide", True, None, 1e30, 0, 0.9, 0.9), (70001, 1, F32, 0, "normal", True, 0.5, 0.7, 6, 0.95, 0.01),
]


@pytest.mark.parametrize("rows,pad,dtype,offset,kind,mask,share,temperature,top_k,top_p,min_p", DRAWS)
def test_actions(B, rows, pad, dtype, offset, kind, mask, share, temperature, top_k, top_p, min_p):
    _say("actions", rows, pad, dtype, offset, kind, mask, share, temperature, top_k, top_p, min_p)
    rng = np.random.default_rng(rows + top_k)
    whole, logits = _logits(rng, rows, pad, dtype, kind, offset)
    kept = whole.clone()
    am = (rng.random(rows) < 0.5).astype(np.uint8) * 3 if mask else None
    on = None if share is None else (rng.random(rows) < share).astype(np.uint8) * 2
    u = _uniform(rng, rows)
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    actions = torch.full((rows + 5,), 99, dtype=torch.uint8, device=DEV)
    lp = torch.full((rows + 5,), 99.0, device=DEV)
    how = B.TabxSampling(temperature, top_k, top_p, min_p)
    B.tabx_sample_actions(logits, how, dev(u), actions[:rows], lp[:rows], dev(am), dev(on))
    alone = torch.full((rows,), 99, dtype=torch.uint8, device=DEV)
    B.tabx_sample_actions(logits, how, dev(u), alone, None, dev(am), dev(on))
    got = actions.cpu().numpy()
    assert (got[rows:] == 99).all() and bool((lp[rows:] == 99).all())
    assert np.array_equal(alone.cpu().numpy(), got[:rows])
    assert torch.equal(whole.view(torch.uint8), kept.view(torch.uint8))
    l = R.allowed(R.f64(logits), am)
    want = np.full(rows, 99)
    for r in range(rows):
        if on is None or on[r]:
            c = R.choose(l[r], temperature, top_k, top_p, min_p, u[r])
            want[r] = 0 if c is None else c
    bad = np.nonzero(got[:rows] != want)[0]
    assert bad.size == 0, (bad[:5], l[bad[:3]], u[bad[:3]], got[bad[:3]], want[bad[:3]])
    sel = np.ones(rows, bool) if on is None else on != 0
    if temperature == 0.0:
        assert (lp.cpu().numpy()[:rows][sel] == 0).all()
    else:
        some = np.minimum(want, 7)
        w_lp, _, b_lp, _ = R.log_prob(l, some, temperature)
        R.near(R.f64(lp)[:rows][sel], w_lp[sel], b_lp[sel], "log_prob")
    assert bool((lp.cpu()[:rows][~torch.from_numpy(sel)] == 99).all())


def test_each_choice_comes_as_often_as_it_should(B):
    """A hundred thousand evenly spaced numbers land in each share to within one of them."""
    n = 100000
    row = torch.tensor([0.1, -1.0, 2.0, 0.3, -2.0, 1.0, 0.0, 0.7], device=DEV)
    logits = row.repeat(n, 1)
    u = ((torch.arange(n, device=DEV, dtype=torch.float64) + 0.5) / n).float()
    actions = torch.empty(n, dtype=torch.uint8, device=DEV)
    B.tabx_sample_actions(logits, B.TabxSampling(), u, actions)
    got = torch.bincount(actions.long(), minlength=8).cpu().numpy()
    want = torch.softmax(row.double(), 0).cpu().numpy() * n
    assert np.abs(got - want).max() <= 1.5, (got, want)


# (rows, pad, type, offset, kind, mask, share, temperature)
PROBS = [
    (1, 0, F32, 0, "normal", False, None, 1.0), (96, 0, F32, 0, "normal", True, None, 1.0),
    (257, 1, F16, 1, "odd", True, 0.5, 1.3), (1000, 0, BF16, 0, "odd", True, None, 0.7),
    (1000, 1, F32, 3, "odd", True, 0.5, 1.0), (4000, 0, F32, 0, "wide", True, 0.5, 1.0),
    (4000, 0, F32, 0, "equal", True, None, 5.0), (333, 8, BF16, 1, "coarse", False, 0.0, 1.0),
    (500, 0, F32, 0, "normal", True, None, 1e-30), (500, 0, F32, 0, "wide", True, None, 1e30),
    (70001, 0, F32, 0, "normal", True, 0.5, 1.0), (5003, 2, F16, 0, "normal", True, None, 0.3),
]


@pytest.mark.parametrize("rows,pad,dtype,offset,kind,mask,share,temperature", PROBS)
def test_log_prob_and_gradient(B, rows, pad, dtype, offset, kind, mask, share, temperature):
    _say("log prob", rows, pad, dtype, offset, kind, mask, share, temperature)
    rng = np.random.default_rng(rows)
    whole, logits = _logits(rng, rows, pad, dtype, kind, offset)
    am = (rng.random(rows) < 0.5).astype(np.uint8) if mask else None
    on = None if share is None else (rng.random(rows) < share).astype(np.uint8)
    acts = rng.integers(0, 8, rows).astype(np.uint8)           # some of them not allowed
    acts[::17] = 200
    gl, ge = rng.normal(size=rows).astype(np.float32), rng.normal(size=rows).astype(np.float32)
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    lp, h = torch.full((rows,), 99.0, device=DEV), torch.full((rows,), 99.0, device=DEV)
    B.tabx_action_log_prob(logits, dev(acts), temperature, lp, h, dev(am), dev(on))
    lp2 = torch.full((rows,), 99.0, device=DEV)
    B.tabx_action_log_prob(logits, dev(acts), temperature, lp2, None, dev(am), dev(on))
    assert torch.equal(lp, lp2)
    sel = np.ones(rows, bool) if on is None else on != 0
    l = R.allowed(R.f64(logits), am)
    w_lp, w_h, b_lp, b_h = R.log_prob(l, acts, temperature)
    R.near(R.f64(lp)[sel], w_lp[sel], b_lp[sel], "log_prob")
    R.near(R.f64(h)[sel], w_h[sel], b_h[sel], "entropy")
    assert (R.f64(lp)[~sel] == 99).all() and (R.f64(h)[~sel] == 99).all()
    for kind_of in ("both", "log_prob", "entropy"):
        a, b = (gl if kind_of != "entropy" else np.zeros_like(gl)), (ge if kind_of != "log_prob" else np.zeros_like(ge))
        out, view = _logits(rng, rows, pad, dtype, "normal", offset)
        B.tabx_action_log_prob_backward(logits, dev(acts), temperature, dev(gl) if kind_of != "entropy" else None,
                                        dev(ge) if kind_of != "log_prob" else None, view, dev(am), dev(on))
        w_g, b_g = R.log_prob_grad(l, acts, temperature, a.astype(np.float64), b.astype(np.float64), dtype)
        R.near(R.f64(view)[sel], w_g[sel], b_g[sel], "grad_logits " + kind_of)
        assert (R.f64(view)[~sel] == 0).all()
        left = torch.ones_like(out, dtype=torch.bool)
        left.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
        assert bool((out[left] == 7).all())
    # in place
    same = torch.empty_like(logits.contiguous())
    B.tabx_action_log_prob_backward(logits, dev(acts), temperature, dev(gl), dev(ge), same, dev(am), dev(on))
    B.tabx_action_log_prob_backward(logits, dev(acts), temperature, dev(gl), dev(ge), logits, dev(am), dev(on))
    assert torch.equal(logits, same)


def test_gradient_against_differences(B):
    rng = np.random.default_rng(3)
    rows, t = 64, 0.9
    z = torch.from_numpy(rng.normal(size=(rows, 8))).float().to(DEV)
    acts = torch.from_numpy(rng.integers(0, 8, rows).astype(np.uint8)).to(DEV)
    gl, ge = torch.from_numpy(rng.normal(size=(2, rows))).float().to(DEV)
    g = torch.empty_like(z)
    B.tabx_action_log_prob_backward(z, acts, t, gl, ge, g)
    d = torch.from_numpy(rng.normal(size=(rows, 8))).float().to(DEV)
    h, out = 2.0 ** -7, []
    for sign in (1, -1):
        lp, en = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        B.tabx_action_log_prob(z + sign * h * d, acts, t, lp, en)
        out.append((lp.double() * gl.double() + en.double() * ge.double()))
    slope = (out[0] - out[1]) / (2 * h)
    want = (g.double() * d.double()).sum(1)
    # third derivative of a log-sum of eight exponentials along d: at most 6 (max |d| / t)^3; an
    # entropy's is at most 20 times that with its logarithms below 6; results below 8 in size
    third = (6 * gl.double().abs() + 120 * ge.double().abs()) * (d.double().abs().amax(1) / t) ** 3
    rounding = 16 * 2.0 ** -24 * 8 * (gl.double().abs() + ge.double().abs()) / h
    assert bool(((slope - want).abs() <= third * h * h / 6 + rounding).all())


def test_a_drawn_action_has_the_log_prob_that_is_evaluated(B):
    rng = np.random.default_rng(5)
    rows = 5000
    for dtype in (F32, BF16, F16):
        _, z = _logits(rng, rows, 1, dtype, "normal")
        am = torch.from_numpy((rng.random(rows) < 0.5).astype(np.uint8)).to(DEV)
        u = torch.from_numpy(rng.random(rows)).float().to(DEV)
        a, lp, lp2 = torch.empty(rows, dtype=torch.uint8, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        B.tabx_sample_actions(z, B.TabxSampling(0.8, 4, 0.9, 0.01), u, a, lp, am)
        B.tabx_action_log_prob(z, a, 0.8, lp2, None, am)
        assert torch.equal(lp, lp2)                             # so that the first ratio is one
        assert not bool(((a == 5) & (am == 0)).any())


# (envs, levels, per-env table pad or None for one table, type, kind, level mask, env mask, t, k, p, m)
LEVELS = [
    (1, 1, None, F32, "normal", False, False, 1.0, 0, 1.0, 0.0), (70, 2, None, F32, "normal", False, True, 1.0, 1, 1.0, 0.0),
    (5003, 257, None, F32, "normal", True, True, 0.5, 0, 1.0, 0.0), (300, 3, 0, BF16, "normal", True, True, 1.0, 0, 0.9, 0.0),
    (50, 5, 2, F32, "odd", False, False, 1.0, 0, 1.0, 0.0), (1000, 255, None, BF16, "coarse", False, False, 0.7, 40, 1.0, 0.0),
    (1025, 256, None, F32, "coarse", True, True, 1.0, 100, 0.8, 0.01), (2000, 1000, None, F16, "equal", False, False, 1.0, 0, 0.5, 0.0),
    (2000, 1000, None, F32, "equal", True, True, 1.0, 333, 0.25, 1.0), (513, 1023, None, F32, "normal", False, True, 0.3, 1022, 1.0, 0.0),
    (513, 1024, None, F32, "normal", True, False, 0.3, 0, 0.3, 0.0), (513, 1025, None, F32, "normal", True, True, 0.3, 7, 0.9, 0.0),
    (3000, 4096, None, F32, "normal", True, True, 0.3, 1000, 0.95, 0.001), (200, 4095, None, BF16, "coarse", False, False, 1.0, 2000, 0.9, 0.0),
    (300, 4097, None, F32, "odd", True, True, 2.0, 3000, 0.99, 0.0), (300, 8191, None, F32, "coarse", True, True, 0.1, 0, 0.6, 0.0),
    (300, 8192, None, F16, "normal", False, False, 1.0, 0, 1.0, 0.1), (300, 8193, None, F32, "normal", True, True, 1.0, 5000, 0.9, 1e-3),
    (2100, 16383, None, BF16, "coarse", True, True, 1.0, 9999, 0.7, 0.0), (300, 16384, None, F32, "equal", False, False, 1.0, 0, 0.75, 0.0),
    (300, 16384, None, F32, "wide", True, True, 0.5, 0, 0.999, 0.0), (40, 700, 1, F16, "coarse", True, True, 0.9, 300, 0.9, 0.0),
    (21, 2048, 0, F32, "odd", True, True, 1.0, 0, 0.95, 0.0), (9, 6001, 3, BF16, "normal", False, True, 1.0, 50, 0.9, 0.0),
    (5, 12000, 0, F32, "normal", True, False, 1.0, 0, 1.0, 0.0), (300, 900, None, F32, "coarse", True, True, 0.0, 0, 1.0, 0.0),
    (30, 5000, 1, F32, "odd", True, True, 0.0, 5, 0.5, 0.0), (64, 300, None, F32, "normal", True, True, 1e-30, 0, 0.9, 0.0),
    (64, 300, None, F32, "wide", True, True, 1e30, 0, 0.9, 0.0), (400, 600, None, F32, "normal", True, True, 1.0, 600, 1.0, 0.0),
    (400, 600, None, F32, "normal", True, True, 1.0, 2 ** 31 - 1, 1e-7, 0.0),
    (300, 1000, None, F32, "cluster", True, True, 30.0, 500, 1.0, 0.0), (300, 4096, None, F32, "cluster", False, True, 30.0, 0, 0.7, 0.0),
    (300, 4000, None, F32, "cluster", True, True, 1.0, 3, 0.9, 0.0), (300, 8000, None, F16, "cluster", True, True, 20.0, 4000, 0.6, 0.0),
    (300, 16000, None, F32, "cluster", True, True, 30.0, 7000, 0.8, 1e-3), (9, 4096, 1, F32, "cluster", True, True, 30.0, 2222, 0.8, 0.0),
    (7, 3000, 0, BF16, "coarse", True, True, 1.0, 700, 0.6, 0.0), (7, 1500, 0, F32, "normal", True, True, 1.0, 700, 0.6, 0.0),
    (66000, 300, None, F32, "normal", True, True, 1.0, 70, 0.6, 0.0), (20, 1024, 0, F32, "equal", False, False, 1.0, 300, 0.5, 0.0),
    (300, 2000, None, F32, "normal", True, True, 0.001, 1500, 0.9999, 0.0),
]


@pytest.mark.parametrize("envs,levels,pad,dtype,kind,lmask,emask,temperature,top_k,top_p,min_p", LEVELS)
def test_levels(B, envs, levels, pad, dtype, kind, lmask, emask, temperature, top_k, top_p, min_p):
    _say("levels", envs, levels, pad, dtype, kind, lmask, emask, temperature, top_k, top_p, min_p)
    rng = np.random.default_rng(envs + levels)
    rows = 1 if pad is None else envs
    v = rng.normal(size=(rows, levels)) * 1.5
    if kind == "coarse":
        v = np.round(v * 2) / 2
    elif kind == "equal":
        v[:] = -2.0
    elif kind == "wide":
        v *= 20.0
    elif kind == "cluster":                    # nearly all levels within a sliver of the scores' range
        v *= 1e-3
        v[:, :: max(1, levels // 3)] += 50.0
    elif kind == "odd":
        at = rng.random(v.shape)
        v[at < 0.1] = -INF
        v[(at > 0.1) & (at < 0.2)] = np.nan
        v[(at > 0.2) & (at < 0.3)] = LOWEST[dtype]
        v[rng.random(rows) < 0.2] = -INF
        v[rng.random(rows) < 0.1, levels // 2] = INF
        v[rng.random(rows) < 0.1] = LOWEST[dtype]
    scores = torch.full((rows, levels + (pad or 0)), 7.0, dtype=dtype, device=DEV)[:, :levels]
    scores.copy_(torch.from_numpy(v))
    lm = (rng.random(levels) < 0.8).astype(np.uint8) if lmask else None
    em = (rng.random(envs) < 0.6).astype(np.uint8) if emask else None
    u = _uniform(rng, envs)
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    nxt = torch.full((envs + 3,), -5, dtype=torch.int32, device=DEV)
    how = B.TabxSampling(temperature, top_k, top_p, min_p)
    B.tabx_sample_levels(scores[0] if pad is None else scores, how, dev(u), nxt[:envs], dev(lm), dev(em))
    got = nxt.cpu().numpy()
    assert (got[envs:] == -5).all()
    l = R.f64(scores).copy()
    l[np.isnan(l)] = -INF
    if lm is not None:
        l[:, lm == 0] = -INF
    want = np.full(envs, -5)
    for e in range(envs):
        if em is None or em[e]:
            c = R.choose(l[0 if pad is None else e], temperature, top_k, top_p, min_p, u[e])
            want[e] = -5 if c is None else c
    bad = np.nonzero(got[:envs] != want)[0]
    assert bad.size == 0, (bad.size, bad[:5], u[bad[:5]], got[bad[:5]], want[bad[:5]])


def test_nothing_to_draw_leaves_the_levels(B):
    nxt = torch.arange(70, dtype=torch.int32, device=DEV)
    u = torch.rand(70, device=DEV)
    for s in (torch.full((2000,), -INF, device=DEV), torch.full((9,), float("nan"), device=DEV)):
        for t in (0.0, 1.0):
            B.tabx_sample_levels(s, B.TabxSampling(t), u, nxt)
    none = torch.zeros(5000, dtype=torch.uint8, device=DEV)
    B.tabx_sample_levels(torch.zeros(5000, device=DEV), B.TabxSampling(1.0, 5), u, nxt, none)
    B.tabx_sample_levels(torch.zeros(70, 30, device=DEV), B.TabxSampling(), u, nxt, None, torch.zeros(70, dtype=torch.uint8, device=DEV))
    assert torch.equal(nxt.cpu(), torch.arange(70, dtype=torch.int32))


def test_far_rows(B):
    """Tables and logits whose offsets pass 32 bits."""
    rng = np.random.default_rng(11)
    stride, rows = 1 << 21, 2050
    whole = torch.empty(rows * stride, dtype=BF16, device=DEV).view(rows, stride)
    v = torch.from_numpy(rng.normal(size=(rows, 600))).to(DEV).to(BF16)
    whole[:, :600] = v
    u = torch.from_numpy(rng.random(rows)).float().to(DEV)
    far, near = (torch.zeros(rows, dtype=torch.int32, device=DEV) for _ in range(2))
    B.tabx_sample_levels(whole[:, :600], B.TabxSampling(1.0, 50, 0.9), u, far)
    B.tabx_sample_levels(v, B.TabxSampling(1.0, 50, 0.9), u, near)
    assert torch.equal(far, near)
    a, b = (torch.zeros(rows, dtype=torch.uint8, device=DEV) for _ in range(2))
    p, q = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    B.tabx_sample_actions(whole[:, :8], B.TabxSampling(), u, a, p)
    B.tabx_sample_actions(v[:, :8], B.TabxSampling(), u, b, q)
    assert torch.equal(a, b) and torch.equal(p, q)
    g = torch.empty(rows, 8, dtype=BF16, device=DEV)
    B.tabx_action_log_prob_backward(v[:, :8], a, 1.0, u, u, g)
    B.tabx_action_log_prob_backward(whole[:, :8], a, 1.0, u, u, whole[:, 8:16])
    assert torch.equal(whole[:, 8:16], g)
