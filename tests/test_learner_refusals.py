"""Which of the learner's calls are refused, on the host: nothing here reaches a GPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import build
    if build.is_stale():
        build.build()
    from paper_2602_01665_amd import binding
    return binding


FAKE = 0x100000          # an address that is only looked at


def _rows(B, stride, type=0, data=FAKE):
    return C.byref(B.TabxRows(data, stride, type))


def _or(given, default):
    """What was given; NULL for 0, the default for None."""
    return default if given is None else (None if isinstance(given, int) else given)


def _norm(B, rows=4, width=8, x=None, y=None, eps=1e-5, mean=FAKE, rstd=FAKE, weight=FAKE, bias=FAKE):
    x = _or(x, _rows(B, width))
    y = _or(y, _rows(B, width))
    return B._lib.tabx_layer_norm(rows, width, x, None, weight, bias, eps, y, mean, rstd, None)


def test_layer_norm_arguments(B):
    nan, inf = float("nan"), float("inf")
    assert _norm(B, rows=0, x=0, y=0) == 0                       # nothing to do, nothing needed
    for kw in (dict(rows=-1), dict(rows=(1 << 40) + 1), dict(width=0), dict(width=-3),
               dict(width=B_MAX + 1), dict(x=_rows(B, 7)), dict(y=_rows(B, 7)),
               dict(x=_rows(B, 8, 3)), dict(y=_rows(B, 8, -1)), dict(rows=1 << 30, x=_rows(B, 1 << 33))):
        assert _norm(B, **kw) == -2, kw
    for kw in (dict(eps=-1e-9), dict(eps=nan), dict(eps=inf)):
        assert _norm(B, **kw) == -5, kw
    for kw in (dict(x=0), dict(y=0), dict(x=_rows(B, 8, 0, 0)), dict(mean=None), dict(rstd=None)):
        assert _norm(B, **kw) == -1, kw
    for kw in (dict(x=_rows(B, 8, 0, FAKE + 2)), dict(y=_rows(B, 8, 1, FAKE + 1)), dict(weight=FAKE + 1),
               dict(bias=FAKE + 2), dict(mean=FAKE + 1), dict(rstd=FAKE + 3)):
        assert _norm(B, **kw) == -3, kw


B_MAX = 8192


def _grad(B, rows=64, width=8, grad_x=0, gw=FAKE, gb=FAKE, ws=FAKE, size=None, mean=FAKE, rstd=FAKE, gy=None):
    size = B._lib.tabx_layer_norm_workspace(rows, width) if size is None else size
    gy = _or(gy, _rows(B, width))
    return B._lib.tabx_layer_norm_backward(rows, width, _rows(B, width), None, None, mean, rstd, gy, _or(grad_x, None),
                                           gw, gb, ws, size, None)


def test_layer_norm_backward_arguments(B):
    need = B.tabx_layer_norm_workspace
    assert need(0, 8) > 0 and need(1, 1) >= 8
    # two sums of a row per workgroup, and never more than 1024 workgroups
    assert need(1 << 30, 368) == need(1 << 24, 368) <= 1024 * 2 * 368 * 4
    for rows, width in ((-1, 8), (4, 0), (4, B_MAX + 1)):
        assert B._lib.tabx_layer_norm_workspace(rows, width) == -2
        with pytest.raises(B.TabxError):
            need(rows, width)
    assert _grad(B, rows=0, gw=None, gb=None, ws=None, mean=None, gy=0) == 0
    for kw in (dict(rows=-1), dict(width=0), dict(size=need(64, 8) - 1), dict(grad_x=_rows(B, 7)), dict(gy=_rows(B, 8, 9))):
        assert _grad(B, **dict(dict(size=1 << 20), **kw)) == -2, kw
    for kw in (dict(ws=None), dict(gw=None, gb=None), dict(mean=None), dict(rstd=None), dict(gy=0)):
        assert _grad(B, **kw) == -1, kw
    for kw in (dict(ws=FAKE + 8), dict(gw=FAKE + 1), dict(gb=FAKE + 2), dict(mean=FAKE + 2)):
        assert _grad(B, **kw) == -3, kw


BAD_SAMPLING = [dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                dict(temperature=1e-31), dict(temperature=1e31), dict(top_k=-1), dict(top_p=0.0),
                dict(top_p=1.5), dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1),
                dict(min_p=float("nan"))]


def test_sampling_arguments(B):
    def act(rows=4, logits=None, how=None, uniform=FAKE, actions=FAKE, lp=FAKE):
        logits = _or(logits, _rows(B, 8))
        how = _or(how, C.byref(B.TabxSampling()))
        return B._lib.tabx_sample_actions(rows, logits, None, None, how, uniform, actions, lp, None)

    def lev(envs=4, levels=8, scores=None, how=None, uniform=FAKE, out=FAKE):
        scores = _or(scores, _rows(B, 0))
        how = _or(how, C.byref(B.TabxSampling()))
        return B._lib.tabx_sample_levels(envs, levels, scores, None, None, how, uniform, out, None)

    assert act(rows=0, logits=0, uniform=None, actions=None) == 0
    assert lev(envs=0, scores=0, uniform=None, out=None) == 0
    for kw in BAD_SAMPLING:
        how = C.byref(B.TabxSampling(**kw))
        assert act(how=how) == -5 and lev(how=how) == -5, kw
    assert act(how=0) == -1 and lev(how=0) == -1
    for kw in (dict(rows=-1), dict(logits=_rows(B, 7)), dict(logits=_rows(B, 0)), dict(logits=_rows(B, 8, 5))):
        assert act(**kw) == -2, kw
    for kw in (dict(logits=0), dict(logits=_rows(B, 8, 0, None)), dict(uniform=None), dict(actions=None)):
        assert act(**kw) == -1, kw
    for kw in (dict(logits=_rows(B, 8, 0, FAKE + 2)), dict(uniform=FAKE + 1), dict(lp=FAKE + 2)):
        assert act(**kw) == -3, kw
    for kw in (dict(envs=-1), dict(envs=(1 << 30) + 1), dict(levels=0), dict(levels=16385),
               dict(scores=_rows(B, 7)), dict(scores=_rows(B, -8)), dict(scores=_rows(B, 0, 4))):
        assert lev(**kw) == -2, kw
    for kw in (dict(scores=0), dict(uniform=None), dict(out=None)):
        assert lev(**kw) == -1, kw
    for kw in (dict(scores=_rows(B, 0, 1, FAKE + 1)), dict(out=FAKE + 2)):
        assert lev(**kw) == -3, kw


def test_log_prob_arguments(B):
    def fwd(rows=4, logits=None, actions=FAKE, t=1.0, lp=FAKE, h=FAKE):
        logits = _or(logits, _rows(B, 8))
        return B._lib.tabx_action_log_prob(rows, logits, None, None, actions, t, lp, h, None)

    def bwd(rows=4, t=1.0, actions=FAKE, gl=FAKE, ge=FAKE, out=None):
        out = _or(out, _rows(B, 8))
        return B._lib.tabx_action_log_prob_backward(rows, _rows(B, 8), None, None, actions, t, gl, ge, out, None)

    assert fwd(rows=0, logits=0, actions=None, lp=None) == 0 and bwd(rows=0, actions=None, out=0) == 0
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-31):
        assert fwd(t=t) == -5 and bwd(t=t) == -5
    assert fwd(rows=-1) == -2 and bwd(out=_rows(B, 7)) == -2 and bwd(out=_rows(B, 8, 3)) == -2
    for rc in (fwd(logits=0), fwd(actions=None), fwd(lp=None), bwd(gl=None, ge=None), bwd(out=0), bwd(actions=None)):
        assert rc == -1
    for rc in (fwd(lp=FAKE + 2), fwd(h=FAKE + 1), bwd(gl=FAKE + 1), bwd(ge=FAKE + 3), bwd(out=_rows(B, 8, 1, FAKE + 1))):
        assert rc == -3


def test_tensors_are_checked_before_their_addresses_are_taken(B):
    """The Python calls refuse a wrong type, size or layout, and host memory."""
    f, u8 = torch.float32, torch.uint8
    x, y = torch.zeros(6, 16), torch.zeros(6, 16)
    w, r = torch.ones(16), torch.zeros(6)

    def refused(why, call, *args, **kw):
        with pytest.raises(B.TabxError, match=why):
            call(*args, **kw)

    norm = B.tabx_layer_norm
    refused("not on a GPU", norm, x, w, w, 1e-5, y, r, r)
    refused("not one of", norm, x.double(), w, w, 1e-5, y)
    refused("not one of", norm, x, w, w, 1e-5, y.to(torch.int32))
    refused("no dimensions", norm, torch.zeros(()), w, w, 1e-5, y)
    refused("rows of 15", norm, x, w, w, 1e-5, y[:, :15])
    refused("y has 5 rows", norm, x, w, w, 1e-5, y[:5])
    refused("next to each other", norm, torch.zeros(16, 6).t(), w, w, 1e-5, y)
    refused("overlap", norm, torch.zeros(1, 16).expand(6, 16), w, w, 1e-5, y)
    refused("equal distances", norm, torch.zeros(3, 4, 16)[:, :2], w, w, 1e-5, y)
    refused("15 elements", norm, x, w[:15], w, 1e-5, y)
    refused("float64", norm, x, w.double(), w, 1e-5, y)
    refused("not contiguous", norm, x, w, torch.zeros(32)[::2], 1e-5, y)
    refused("row_mask", norm, x, w, w, 1e-5, y, r, r, torch.zeros(6, dtype=torch.bool))
    grad, ws = B.tabx_layer_norm_backward, torch.zeros(1 << 12, dtype=u8)
    refused("not on a GPU", grad, x, w, r, r, y, None, w, w, ws)
    refused("mean is needed", grad, x, w, None, r, y, None, w, w, ws)
    refused("workspace is", grad, x, w, r, r, y, None, w, w, ws.float())
    refused("grad_y has 5 rows", grad, x, w, r, r, y[:5], None, w, w, ws)
    refused("grad_x has 5 rows", grad, x, w, r, r, y, y[:5], w, w, ws)
    lg, how = torch.zeros(6, 8), B.TabxSampling()
    acts, u = torch.zeros(6, dtype=u8), torch.zeros(6)
    refused("not on a GPU", B.tabx_sample_actions, lg, how, u, acts)
    refused("rows of 7", B.tabx_sample_actions, lg[:, :7], how, u, acts)
    refused("uniform has 5", B.tabx_sample_actions, lg, how, u[:5], acts)
    refused("uniform is needed", B.tabx_sample_actions, lg, how, None, acts)
    refused("actions is torch.int64", B.tabx_sample_actions, lg, how, u, acts.long())
    refused("controlled has 3", B.tabx_sample_actions, lg, how, u, acts, None, None, acts[:3])
    nxt = torch.zeros(6, dtype=torch.int32)
    refused("not on a GPU", B.tabx_sample_levels, torch.zeros(9), how, u, nxt)
    refused("scores has 5 rows", B.tabx_sample_levels, torch.zeros(5, 9), how, u, nxt)
    refused("scores has 5 rows", B.tabx_sample_levels, torch.zeros(1, 9).expand(5, 9), how, u, nxt)
    refused("level_mask has 8", B.tabx_sample_levels, torch.zeros(9), how, u, nxt, torch.zeros(8, dtype=u8))
    refused("next_level is torch.int64", B.tabx_sample_levels, torch.zeros(9), how, u, nxt.long())
    refused("not on a GPU", B.tabx_action_log_prob, lg, acts, 1.0, u)
    refused("log_prob is needed", B.tabx_action_log_prob, lg, acts, 1.0, None)
    refused("not on a GPU", B.tabx_action_log_prob_backward, lg, acts, 1.0, u, u, lg)
    refused("grad_logits has 5", B.tabx_action_log_prob_backward, lg, acts, 1.0, u, u, lg[:5])
    assert f is x.dtype


def test_a_batch_refuses_draws_that_would_mean_something_else(B):
    """Actions without the observation's mask; levels without a bank, or out of another number of them."""
    from paper_2602_01665_amd import inputs as I
    w = I.WORKLOADS["c2_4096env_5v5"]

    def env(E, **kw):
        over = {k: kw.pop(k) for k in ("num_levels",) if k in kw}
        return B.TabxEnv(I.make_params(w, E, **over), I.make_scenario(w, over.get("num_levels", E)), device="cpu", **kw)

    how, u = B.TabxSampling(), torch.zeros(4)
    one = env(4, want_action_mask=False)
    acts = torch.zeros(4, one.N, dtype=torch.uint8)
    logits = torch.zeros(4, one.N, 8)
    for batch in [one] + one.parts(1):
        with pytest.raises(B.TabxError, match="no action mask"):
            batch.sample_actions(logits, how, torch.zeros(4, one.N), acts)
        with pytest.raises(B.TabxError, match="no bank of levels"):
            batch.sample_levels(torch.zeros(3), how, u)
    bank = env(4, num_levels=6)
    for batch in [bank] + bank.parts(1):
        for wrong in (torch.zeros(5), torch.zeros(7), torch.zeros(4, 12)):
            with pytest.raises(B.TabxError, match="not 6"):
                batch.sample_levels(wrong, how, u)
        with pytest.raises(B.TabxError, match="no dimensions"):
            batch.sample_levels(torch.zeros(()), how, u)
        with pytest.raises(B.TabxError, match="not on a GPU"):      # what is left to refuse on the host
            batch.sample_levels(torch.zeros(6), how, u)
        with pytest.raises(B.TabxError, match="not on a GPU"):
            batch.sample_actions(logits, how, torch.zeros(4, one.N), acts)


def test_sizes_that_32_bits_do_not_hold_are_not_cut_off(B):
    wide = torch.empty(2, 2 ** 32 + 8, device="meta")
    x, how, u8 = torch.zeros(2, 8), B.TabxSampling(), torch.zeros(2, dtype=torch.uint8)

    def refused(call, *args):
        with pytest.raises(B.TabxError, match="rows of 4294967304"):
            call(*args)

    refused(B.tabx_layer_norm, wide, None, None, 1e-5, wide)
    refused(B.tabx_layer_norm, x, None, None, 1e-5, wide)
    refused(B.tabx_layer_norm_backward, wide, None, x[:, 0], x[:, 0], wide, wide)
    refused(B.tabx_layer_norm_workspace, 2, 2 ** 32 + 8)
    refused(B.tabx_sample_levels, wide, how, x[:, 0], torch.zeros(2, dtype=torch.int32))
    refused(B.tabx_sample_levels, wide[0], how, x[:, 0], torch.zeros(2, dtype=torch.int32))
    refused(B.tabx_sample_actions, wide, how, x[:, 0], u8)
    assert B.TabxSampling(1.0, 2 ** 32 + 5).top_k == 2 ** 31 - 1 and B.TabxSampling(1.0, 5).top_k == 5
    assert B.TabxSampling(1.0, -2 ** 32 + 5).top_k < 0            # refused by every call
    assert B.tabx_layer_norm_workspace(2 ** 40, 8) > 0
    for rows in (2 ** 64 + 4, 2 ** 63, -2 ** 64 + 4):
        with pytest.raises(B.TabxError):
            B.tabx_layer_norm_workspace(rows, 8)
