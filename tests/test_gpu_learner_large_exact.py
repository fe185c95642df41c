"""Large calls against 64-bit formulas: some rows at the start, in the middle and at the end of draws and
log-probabilities and of a layer norm's gradient, and its sums over all rows (needs an MI355X)."""
import numpy as np
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


def _some(rows, n=400):
    return torch.cat([torch.arange(a, a + n) for a in (0, rows // 2, rows - n)]).to(DEV)


@pytest.mark.parametrize("dtype,pad,how", [(F32, 0, (0.8, 6, 0.9, 0.01)), (BF16, 1, (1.0, 0, 1.0, 0.0)), (F16, 0, (1.3, 0, 0.9999, 1e-5))])
def test_choices(B, dtype, pad, how):
    rows = 1100003
    print("[gpu] choices", dtype, pad, how, flush=True)
    g = torch.Generator(device=DEV).manual_seed(6)
    z = (2.0 * torch.randn(rows, 8 + pad, generator=g, device=DEV)).to(dtype)[:, :8]
    u = torch.rand(rows, generator=g, device=DEV)
    mask, on = (torch.rand(2, rows, generator=g, device=DEV) < 0.5).to(torch.uint8)
    gl, ge = torch.randn(2, rows, generator=g, device=DEV)
    a, lp, h = torch.full((rows,), 99, dtype=torch.uint8, device=DEV), torch.full((rows,), 99.0, device=DEV), torch.full((rows,), 99.0, device=DEV)
    grad = torch.ones(rows, 8 + pad, device=DEV).to(dtype)[:, :8]
    B.tabx_sample_actions(z, B.TabxSampling(*how), u, a, lp, mask, on)
    B.tabx_action_log_prob_backward(z, a, how[0], gl, ge, grad, mask, on)
    lp2 = torch.full((rows,), 99.0, device=DEV)
    B.tabx_action_log_prob(z, a, how[0], lp2, h, mask, on)
    assert torch.equal(lp, lp2)
    at = _some(rows)
    c = [R.f64(t[at]) for t in (a, lp, h, grad, u, gl, ge)]
    l, learns = R.allowed(R.f64(z[at]), mask[at].cpu().numpy()), on[at].cpu().numpy() != 0
    want = np.array([R.choose(l[r], *how, c[4][r]) if learns[r] else 99 for r in range(len(l))])
    assert np.array_equal(c[0], want)
    acts = np.where(learns, want, 0).astype(np.uint8)
    w_lp, w_h, b_lp, b_h = R.log_prob(l, acts, how[0])
    R.near(c[1][learns], w_lp[learns], b_lp[learns], "log_prob")
    R.near(c[2][learns], w_h[learns], b_h[learns], "entropy")
    w_g, b_g = R.log_prob_grad(l, acts, how[0], c[5], c[6], dtype)
    R.near(c[3][learns], w_g[learns], b_g[learns], "grad_logits")
    assert (c[3][~learns] == 0).all() and (c[1][~learns] == 99).all()


@pytest.mark.parametrize("rows,width,tx,tg,masked,inputs", [
    (130000, 368, F32, BF16, True, False), (85051, 512, BF16, BF16, False, True), (700001, 16, F32, F32, True, True),
    (40000, 2000, F32, F32, False, False), (6000, 4100, BF16, BF16, True, True), (1500001, 4, F16, F16, True, True)])
def test_layer_norm_backward(B, rows, width, tx, tg, masked, inputs):
    print("[gpu] norm grad", rows, width, tx, tg, masked, inputs, flush=True)
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = (1.0 + 2.0 * torch.randn(rows, width, generator=g, device=DEV)).to(tx)
    gy, w = torch.randn(rows, width, generator=g, device=DEV).to(tg), torch.randn(width, generator=g, device=DEV)
    on = (torch.rand(rows, generator=g, device=DEV) < 0.5).to(torch.uint8) if masked else None
    mean = x.float().mean(1).contiguous()
    rstd = torch.rsqrt(x.float().var(1, unbiased=False) + 1e-5).contiguous()
    gx = torch.full((rows, width), 3.0, device=DEV).to(tx) if inputs else None
    gw, gb = torch.zeros(width, device=DEV), torch.zeros(width, device=DEV)
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    B.tabx_layer_norm_backward(x, w, mean, rstd, gy, gx, gw, gb, ws, on)
    want, size = torch.zeros(2, width, dtype=torch.float64, device=DEV), torch.zeros(2, width, dtype=torch.float64, device=DEV)
    step = max(1, 20000000 // width)
    for a in range(0, rows, step):
        s = slice(a, a + step)
        d = gy[s].double() if on is None else torch.where(on[s, None] != 0, gy[s].double(), 0.0)
        t = d * ((x[s].double() - mean[s, None].double()) * rstd[s, None].double())
        want += torch.stack([t.sum(0), d.sum(0)])
        size += torch.stack([t.abs().sum(0), d.abs().sum(0)])
    # what one lane adds up, at most all rows of its workgroup, and 64 joining additions (as in the tests of few rows)
    groups = B.tabx_layer_norm_workspace(rows, width) // (8 * width)
    chain = (-(-rows // groups) + 64 + 64 + 4) * R.U
    assert bool(((torch.stack([gw, gb]).double() - want).abs() <= chain * size).all())
    if inputs:
        at = _some(rows, 100)
        keep = np.ones(len(at), bool) if on is None else on[at].cpu().numpy() != 0
        wx, _, _, bx, _, _ = R.norm_grad(R.f64(x[at]), keep, R.f64(w), R.f64(mean[at]), R.f64(rstd[at]), R.f64(gy[at]), tx, 1)
        R.near(gx[at], wx, bx, "grad_x")
