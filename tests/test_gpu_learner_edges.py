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
