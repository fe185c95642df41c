"""Calls large enough for what the launches do beyond some size (several runs of rows per team,
results past the caches, inputs read once) against the same calls on a few rows at a time, which the
other tests hold to 64 bits (needs an MI355X)."""
import pytest
import torch

from tests import learner_reference as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def _say(*a):
    print("[gpu]", *a, flush=True)


def _normal(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device=DEV)


def _parts(rows, step):
    return [slice(a, min(rows, a + step)) for a in range(0, rows, step)]


@pytest.mark.parametrize("rows,width,tx,ty,masked", [
    (50000, 368, F32, BF16, True), (30001, 368, F32, F32, False), (50000, 366, BF16, F16, False),
    (400000, 96, F32, BF16, True), (100000, 186, F32, BF16, False), (9000, 2048, F32, BF16, True),
    (5000, 4100, BF16, BF16, True), (3001, 6001, F32, F32, False), (1200001, 16, F32, F32, True),
    (2500000, 7, F16, F16, False), (6000003, 3, F32, F32, True), (60000, 700, BF16, BF16, False),
    (20000, 1300, F32, F16, False),
])
def test_layer_norm(B, rows, width, tx, ty, masked):
    _say("norm", rows, width, tx, ty, masked)
    n = _normal(rows)
    x = (1.0 + 2.0 * n(rows, width)).to(tx)
    w, b = n(width), n(width)
    on = (n(rows) > 0).to(torch.uint8) if masked else None
    whole = [torch.full((rows, width), 3.0, dtype=ty, device=DEV), torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)]
    parts = [t.clone() for t in whole]
    B.tabx_layer_norm(x, w, b, 1e-5, *whole, on)
    for s in _parts(rows, max(64, rows // 13)):
        B.tabx_layer_norm(x[s], w, b, 1e-5, *(t[s] for t in parts), None if on is None else on[s])
    for p, q, what in zip(whole, parts, ("y", "mean", "rstd")):
        assert torch.equal(p, q), what
    few = slice(0, 300)                        # (a check that the parts are not wrong together)
    keep = torch.ones(300, dtype=torch.bool) if on is None else on[few].cpu() != 0
    y, _, _, bound, _, _ = R.norm(R.f64(x[few]), R.f64(w), R.f64(b), 1e-5, ty)
    R.near(R.f64(whole[0][few])[keep], y[keep], bound[keep] + 1e-12, "y")


@pytest.mark.parametrize("rows,width,tx,tg,masked,inputs", [
    (130000, 368, F32, BF16, True, False), (85051, 512, BF16, BF16, False, True), (300001, 40, F32, F32, True, True),
    (20000, 1100, F32, BF16, False, True), (6000, 4100, BF16, BF16, True, True), (3001, 6001, F32, F32, False, True),
    (700001, 16, F32, F32, True, True), (70000, 700, BF16, BF16, False, True), (40000, 2000, F32, F32, False, False),
    (1500001, 4, F16, F16, True, True), (500000, 96, F32, BF16, True, False), (2000000, 30, F32, BF16, False, False),
])
def test_layer_norm_backward(B, rows, width, tx, tg, masked, inputs):
    _say("norm grad", rows, width, tx, tg, masked, inputs)
    n = _normal(rows)
    x, gy, w = (1.0 + 2.0 * n(rows, width)).to(tx), n(rows, width).to(tg), n(width)
    on = (n(rows) > 0).to(torch.uint8) if masked else None
    mean, rstd = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
    B.tabx_layer_norm(x, None, None, 1e-5, torch.empty_like(x), mean, rstd)
    whole = torch.full((rows, width), 3.0, dtype=tx, device=DEV) if inputs else None
    part = whole.clone() if inputs else None
    sums = [torch.zeros(width, device=DEV) for _ in range(2)]
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    B.tabx_layer_norm_backward(x, w, mean, rstd, gy, whole, *sums, ws, on)
    total = [torch.zeros(width, dtype=torch.float64, device=DEV) for _ in range(2)]
    size = [torch.zeros(width, dtype=torch.float64, device=DEV) for _ in range(2)]
    few = [torch.zeros(width, device=DEV) for _ in range(2)]
    for s in _parts(rows, max(64, rows // 13)):
        m = None if on is None else on[s]
        B.tabx_layer_norm_backward(x[s], w, mean[s], rstd[s], gy[s], part[s] if inputs else None, *few, ws, m)
        for t, f in zip(total, few):
            t += f.double()
        a = gy[s].double().abs() if m is None else gy[s].double().abs() * m[:, None].double()
        size[0] += (a * ((x[s].double() - mean[s, None].double()) * rstd[s, None].double()).abs()).sum(0)
        size[1] += a.sum(0)
    if inputs:
        assert torch.equal(whole, part)
    # both sides add at most as many rows one after the other as a lane has, and join them in 64 steps
    groups = B.tabx_layer_norm_workspace(rows, width) // (8 * width)
    chain = 2 * (-(-rows // groups) + 64 + 64 + 8) * R.U
    for got, want, mag in zip(sums, total, size):
        assert bool(((got.double() - want).abs() <= chain * mag).all())


def test_choices(B):
    """More than a million rows: draws, log-probabilities, and a gradient that goes past the caches."""
    rows = 1100003
    n = _normal(5)
    z, u = 2.0 * n(rows, 8), torch.rand(rows, device=DEV)
    mask, on = (n(rows) > 0).to(torch.uint8), (n(rows) > 0).to(torch.uint8)
    how = B.TabxSampling(0.8, 6, 0.9, 0.01)

    def run(s, out):
        B.tabx_sample_actions(z[s], how, u[s], out["a"][s], out["lp"][s], mask[s], on[s])
        B.tabx_action_log_prob(z[s], out["a"][s], 0.8, out["lp2"][s], out["h"][s], mask[s], on[s])
        B.tabx_action_log_prob_backward(z[s], out["a"][s], 0.8, u[s], u[s], out["g"][s], mask[s], on[s])

    def buffers():
        return {"a": torch.zeros(rows, dtype=torch.uint8, device=DEV), "lp": torch.zeros(rows, device=DEV),
                "lp2": torch.zeros(rows, device=DEV), "h": torch.zeros(rows, device=DEV), "g": torch.ones(rows, 8, device=DEV)}

    whole, parts = buffers(), buffers()
    run(slice(0, rows), whole)
    for s in _parts(rows, 99991):
        run(s, parts)
    for k in whole:
        assert torch.equal(whole[k], parts[k]), k
    assert torch.equal(whole["lp"], whole["lp2"])
    assert bool((whole["g"][on == 0] == 0).all())


def test_levels(B):
    """As many envs as fit a call's workgroups several times, and a table for each of many envs."""
    n = _normal(7)
    u = torch.rand(300007, device=DEV)
    scores = n(3000)
    how = B.TabxSampling(0.7, 900, 0.9, 0.001)
    whole, parts = (torch.zeros(300007, dtype=torch.int32, device=DEV) for _ in range(2))
    B.tabx_sample_levels(scores, how, u, whole)
    for s in _parts(300007, 30011):
        B.tabx_sample_levels(scores, how, u[s], parts[s])
    assert torch.equal(whole, parts)
    tables = n(70001, 40)                      # more of them than a grid has columns
    whole, parts = (torch.zeros(70001, dtype=torch.int32, device=DEV) for _ in range(2))
    B.tabx_sample_levels(tables, B.TabxSampling(0.7, 9), u[:70001], whole)
    for s in _parts(70001, 9973):
        B.tabx_sample_levels(tables[s], B.TabxSampling(0.7, 9), u[s], parts[s])
    assert torch.equal(whole, parts)


def test_more_rows_than_32_bits_count(B):
    """2^31 rows and some: the last ones are worked on where they lie."""
    rows, few = 2 ** 31 + 300, 700
    last = slice(rows - few, rows)
    z = torch.zeros(rows, 8, dtype=BF16, device=DEV)
    n = _normal(9)
    z[last] = n(few, 8).to(BF16)
    u = torch.zeros(rows, device=DEV)
    u[last] = torch.rand(few, device=DEV)
    a = torch.zeros(rows, dtype=torch.uint8, device=DEV)
    how = B.TabxSampling(0.9, 5)
    B.tabx_sample_actions(z, how, u, a)
    want = torch.zeros(few, dtype=torch.uint8, device=DEV)
    B.tabx_sample_actions(z[last].clone(), how, u[last].clone(), want)
    assert torch.equal(a[last], want)
    del u
    g, want = torch.ones_like(z), torch.empty(few, 8, dtype=BF16, device=DEV)
    lp = torch.full((rows,), 0.5, device=DEV)
    B.tabx_action_log_prob_backward(z, a, 1.0, lp, None, g)
    B.tabx_action_log_prob_backward(z[last].clone(), a[last].clone(), 1.0, lp[:few].clone(), None, want)
    assert torch.equal(g[last], want)
    B.tabx_action_log_prob(z, a, 1.0, lp)
    want = torch.empty(few, device=DEV)
    B.tabx_action_log_prob(z[last].clone(), a[last].clone(), 1.0, want)
    assert torch.equal(lp[last], want)
    del z, g, a, lp
    torch.cuda.empty_cache()
    x = torch.zeros(rows, 5, dtype=BF16, device=DEV)
    x[last] = n(few, 5).to(BF16)
    w = 1.0 + n(5)
    y, mean, rstd = torch.ones_like(x), torch.ones(rows, device=DEV), torch.ones(rows, device=DEV)
    B.tabx_layer_norm(x, w, None, 1e-5, y, mean, rstd)
    part = [torch.empty(few, 5, dtype=BF16, device=DEV), torch.empty(few, device=DEV), torch.empty(few, device=DEV)]
    B.tabx_layer_norm(x[last].clone(), w, None, 1e-5, *part)
    for p, q in zip((y, mean, rstd), part):
        assert torch.equal(p[last], q)
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, 5), dtype=torch.uint8, device=DEV)
    gw, gx = torch.empty(5, device=DEV), torch.ones_like(x)
    B.tabx_layer_norm_backward(x, w, mean, rstd, y, gx, gw, None, ws)
    want, wx = torch.empty(5, device=DEV), torch.empty(few, 5, dtype=BF16, device=DEV)
    B.tabx_layer_norm_backward(x[last].clone(), w, *part[1:], part[0], wx, want, None, ws)
    assert torch.equal(gx[last], wx)
    # (the other rows are all zero and add exactly nothing)
    h = (x[last].double() - mean[last, None].double()) * rstd[last, None].double()
    mag = (part[0].double() * h).abs().sum(0)
    assert bool(((gw.double() - want.double()).abs() <= 2 * (few + 64 + 64) * R.U * mag).all())
    del x, y, mean, rstd, gx
    torch.cuda.empty_cache()
