"""What the learner's calls promise at their edges: gradients that are not finite, PyTorch's graph around
them (needs an MI355X)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, INF, NAN = "cuda:0", float("inf"), float("nan")


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_that_are_not_finite_stay_with_the_choices_allowed(B, dtype):
    """A choice that is not allowed has a gradient of zero whatever comes back, as have rows that are not
    controlled or have nothing to choose; other rows do not notice."""
    rows = 300
    rng = np.random.default_rng(4)
    z = torch.from_numpy(rng.normal(size=(rows, 8))).to(DEV).to(dtype)
    barred = torch.from_numpy(rng.random((rows, 8)) < 0.3).to(DEV)
    barred[::50] = True
    z[barred] = -INF
    z[3::40, 2], barred[3::40, 2] = NAN, True
    z[7::40, 4], barred[7::40, 4] = INF, False
    mask = torch.from_numpy((rng.random(rows) < 0.5).astype(np.uint8)).to(DEV)
    on = torch.from_numpy((rng.random(rows) < 0.8).astype(np.uint8)).to(DEV)
    barred[:, 5] |= mask == 0
    acts = torch.from_numpy(rng.integers(0, 8, rows).astype(np.uint8)).to(DEV)
    usual = torch.from_numpy(rng.normal(size=(2, rows))).float().to(DEV)
    gl, ge = usual.clone()
    odd = torch.zeros(rows, dtype=torch.bool, device=DEV)
    for k, v in enumerate((NAN, INF, -INF)):
        gl[k::10] = v
        ge[k + 3::10] = v
        gl[k + 6::30], ge[k + 6::30] = v, -v
        odd[k::10], odd[k + 3::10], odd[k + 6::30] = True, True, True
    want, got = torch.empty_like(z), torch.full_like(z, 9.0)
    B.tabx_action_log_prob_backward(z, acts, 0.9, usual[0], usual[1], want, mask, on)
    B.tabx_action_log_prob_backward(z, acts, 0.9, gl, ge, got, mask, on)
    assert bool((got[barred] == 0).all()) and bool((got[on == 0] == 0).all())
    assert torch.equal(got[~odd], want[~odd])
    assert bool(torch.isfinite(want).all())


def test_a_graph_that_needs_what_was_overwritten_is_refused(B):
    """The next tick's rows in the tensor that a network has kept for its backward pass, and the other
    outputs the same: PyTorch refuses that pass, as after a call of its own in place."""
    y, mean, rstd = torch.zeros(6, 16, device=DEV), torch.zeros(6, device=DEV), torch.zeros(6, device=DEV)
    x, m = torch.randn(6, 16, device=DEV), torch.randn(16, 8, device=DEV, requires_grad=True)
    B.tabx_layer_norm(x, None, None, 1e-5, y, mean, rstd)
    out = (y @ m).sum()
    out.backward(retain_graph=True)
    B.tabx_layer_norm(x + 1, None, None, 1e-5, y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()
    (y @ m).sum().backward()


def test_what_each_call_writes_is_told(B):
    f = lambda *s: torch.rand(*s, device=DEV)  # noqa: E731
    e = 40
    x, gy, z, w = f(e, 16), f(e, 16), f(e, 8), f(16)
    acts, nxt = torch.zeros(e, dtype=torch.uint8, device=DEV), torch.zeros(e, dtype=torch.int32, device=DEV)
    o = {k: f(e) for k in ("mean", "rstd", "u", "lp", "h")}
    o.update(y=f(e, 16), gx=f(e, 16), gw=f(16), gb=f(16), gz=f(e, 8), x=x, gy=gy, z=z, w=w, acts=acts, nxt=nxt)
    ws = torch.empty(B.tabx_layer_norm_workspace(e, 16), dtype=torch.uint8, device=DEV)
    how = B.TabxSampling()

    def writes(names, call, *args):
        before = {k: t._version for k, t in o.items()}
        call(*args)
        assert {k for k, t in o.items() if t._version != before[k]} == set(names.split()), names

    writes("y", B.tabx_layer_norm, x, w, None, 1e-5, o["y"])
    writes("y mean rstd", B.tabx_layer_norm, x, w, None, 1e-5, o["y"], o["mean"], o["rstd"])
    writes("gx", B.tabx_layer_norm_backward, x, w, o["mean"], o["rstd"], gy, o["gx"])
    writes("gw gb", B.tabx_layer_norm_backward, x, w, o["mean"], o["rstd"], gy, None, o["gw"], o["gb"], ws)
    writes("acts", B.tabx_sample_actions, z, how, o["u"], acts)
    writes("acts lp", B.tabx_sample_actions, z, how, o["u"], acts, o["lp"])
    writes("nxt", B.tabx_sample_levels, w, how, o["u"], nxt)
    writes("lp h", B.tabx_action_log_prob, z, acts, 1.0, o["lp"], o["h"])
    writes("gz", B.tabx_action_log_prob_backward, z, acts, 1.0, o["lp"], None, o["gz"])
    with torch.inference_mode():               # (whose tensors have no versions)
        B.tabx_layer_norm(x, w, None, 1e-5, f(e, 16))


@pytest.mark.parametrize("rows,width,pad,tx,ty,offset", [
    (100000, 186, 0, torch.float32, torch.float32, 0), (120000, 160, 0, torch.bfloat16, torch.bfloat16, 0),
    (140001, 128, 0, torch.bfloat16, torch.float16, 1), (140001, 128, 32, torch.float32, torch.bfloat16, 32),
    (130001, 130, 0, torch.bfloat16, torch.bfloat16, 0), (300001, 56, 0, torch.float16, torch.bfloat16, 0)])
def test_results_past_the_caches_are_those_of_few_rows(B, rows, width, pad, tx, ty, offset):
    """Rows on and off the boundaries of lines, of one piece and of more."""
    print("[gpu] norm", rows, width, pad, tx, ty, offset, flush=True)
    g = torch.Generator(device=DEV).manual_seed(rows)
    x, w = torch.randn(rows, width, generator=g, device=DEV).to(tx), torch.randn(width, generator=g, device=DEV)
    out = [torch.full((offset + rows * (width + pad),), 3.0, dtype=ty, device=DEV) for _ in range(2)]
    whole, parts = (t[offset:].view(rows, width + pad)[:, :width] for t in out)
    B.tabx_layer_norm(x, w, None, 1e-5, whole)
    for a in range(0, rows, 9000):
        B.tabx_layer_norm(x[a:a + 9000], w, None, 1e-5, parts[a:a + 9000])
    assert torch.equal(*out)
