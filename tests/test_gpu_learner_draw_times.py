"""What a launch of draws takes where many of them are close, against the same launch where few are: the
decisions in 64 bits may not set its time (needs an MI355X)."""
import numpy as np
import pytest
import torch

from tests import learner_reference as R

pytestmark = pytest.mark.gpu
DEV, ROWS = "cuda:0", 655360


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def _time(B, logits, how, u, mask):
    """Microseconds of a launch, the best of five series of twenty in a graph."""
    actions, lp = torch.zeros(ROWS, dtype=torch.uint8, device=DEV), torch.zeros(ROWS, device=DEV)
    B.tabx_sample_actions(logits, how, u, actions, lp, mask)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(20):
            B.tabx_sample_actions(logits, how, u, actions, lp, mask)
    best = float("inf")
    for _ in range(5):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        best = min(best, start.elapsed_time(end) * 1000.0 / 20)
    return best


def _inputs():
    g = torch.Generator(device=DEV).manual_seed(1)
    z = 2.0 * torch.randn(ROWS, 8, generator=g, device=DEV)
    u = torch.rand(ROWS, generator=g, device=DEV)
    return z, u, (torch.rand(ROWS, generator=g, device=DEV) < 0.4).to(torch.uint8)


@pytest.mark.parametrize("close,usual", [
    ((1.0, 0, 1.0, 1e-5), (1.0, 0, 1.0, 0.01)), ((0.3, 0, 1.0, 1e-5), (0.3, 0, 1.0, 0.01)),
    ((0.3, 0, 0.99999, 0.0), (0.3, 0, 0.95, 0.0)), ((1.0, 0, 1e-6, 0.0), (1.0, 0, 0.5, 0.0))])
def test_filters_near_their_ends(B, close, usual):
    """As fast as others (twice is for the noise; with the weights held to an absolute margin, 15 and
    20 times)."""
    z, u, mask = _inputs()
    times = [_time(B, z, B.TabxSampling(*how), u, mask) for how in (close, usual)]
    print("[gpu] draws", close, usual, times, flush=True)
    assert times[0] <= 2.0 * times[1], times


def test_ties(B):
    """Eight equal scores and a top_p of one half: each row's sums are exactly equal.  All of them in 64
    bits, a lane's row in one of eight passes, take seven times as long as a launch without filters
    (in one of 64 passes: 45 times; twelve is between them)."""
    _, u, _ = _inputs()
    z = torch.full((ROWS, 8), 0.25, device=DEV)
    times = [_time(B, z, B.TabxSampling(1.0, 0, p), u, None) for p in (0.5, 1.0)]
    print("[gpu] ties", times, flush=True)
    assert times[0] <= 12.0 * times[1], times


@pytest.mark.parametrize("rows", [1, 63, 1000])
@pytest.mark.parametrize("how", [(1.0, 0, 0.5, 0.0), (0.7, 6, 0.5, 0.5), (1.0, 0, 0.75, 0.0)])
def test_ties_are_right(B, rows, how):
    """Rows of equal scores (of all eight, of four and of none of them) in any order, some of them not
    controlled: each lane gets its own row's draw."""
    rng = np.random.default_rng(rows)
    l = np.full((rows, 8), 0.5, np.float32)
    l[rng.random(rows) < 0.3, ::2] = -np.inf
    l[rng.random(rows) < 0.1] = -np.inf
    l[rng.random((rows, 8)) < 0.05] = 0.25
    u, on = rng.random(rows).astype(np.float32), (rng.random(rows) < 0.7).astype(np.uint8)
    u[::7] = 0.0
    actions = torch.full((rows,), 99, dtype=torch.uint8, device=DEV)
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    B.tabx_sample_actions(dev(l), B.TabxSampling(*how), dev(u), actions, None, None, dev(on))
    want = np.full(rows, 99)
    for r in np.nonzero(on)[0]:
        c = R.choose(l[r].astype(np.float64), *how, u[r])
        want[r] = 0 if c is None else c
    assert np.array_equal(actions.cpu().numpy(), want)
