"""What a launch of draws takes where many of them are close, against the same launch where few are: the
decisions in 64 bits may not set its time (needs an MI355X)."""
import pytest
import torch

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
