"""Layer norm onto its own input, and its gradient onto the one that came in: the bits of the same call
with memory of its own, for every kind of row (needs an MI355X)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda:0"
# one lane a row, 4, 8, 16 (one to three pieces), 32, 64, and workgroups of 128, 256 and 1024; rows enough for several
# turns of every team
WIDTHS = [(1, 70001), (3, 40000), (4, 30000), (13, 30000), (30, 20000), (50, 9000), (96, 9000), (186, 5000), (250, 5000),
          (368, 5000), (515, 4001), (900, 3000), (1026, 3000), (1500, 2000), (2048, 1500), (3001, 1500), (4099, 1400), (6001, 1300), (8192, 1100)]


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def _inputs(rows, width, dtype, masked):
    g = torch.Generator(device=DEV).manual_seed(rows + width)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    on = (n(rows) > 0).to(torch.uint8) if masked else None
    return (1.0 + 2.0 * n(rows, width)).to(dtype), n(rows, width).to(dtype), n(width), n(width), on


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("width,rows", WIDTHS)
def test_forward(B, width, rows, dtype, masked):
    print("[gpu] norm in place", width, rows, dtype, masked, flush=True)
    x, _, w, b, on = _inputs(rows, width, dtype, masked)
    for pad in (0, 3):
        line = torch.full((rows, width + pad), 7.0, dtype=dtype, device=DEV)
        same = line[:, :width]
        same.copy_(x)
        want = x.clone()                       # rows that are masked out keep what is there
        mean, rstd = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
        mean2, rstd2 = mean.clone(), rstd.clone()
        B.tabx_layer_norm(x, w, b, 1e-5, want, mean, rstd, on)
        B.tabx_layer_norm(same, w, b, 1e-5, same, mean2, rstd2, on)
        assert torch.equal(same, want) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
        assert bool((line[:, width:] == 7).all())


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("width,rows", WIDTHS)
def test_backward(B, width, rows, dtype, masked):
    print("[gpu] norm grad in place", width, rows, dtype, masked, flush=True)
    x, gy, w, _, on = _inputs(rows, width, dtype, masked)
    mean = x.float().mean(1).contiguous()
    rstd = torch.rsqrt(x.float().var(1, unbiased=False) + 1e-5).contiguous()
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    sums, sums2 = ([torch.zeros(width, device=DEV) for _ in range(2)] for _ in range(2))
    want, same = torch.full_like(gy, 9.0), gy.clone()
    B.tabx_layer_norm_backward(x, w, mean, rstd, gy, want, *sums, ws, on)
    B.tabx_layer_norm_backward(x, w, mean, rstd, same, same, *sums2, ws, on)
    assert torch.equal(same, want)
    assert all(torch.equal(p, q) for p, q in zip(sums, sums2))
    if masked:
        assert bool((same[on == 0] == 0).all())
    alone = gy.clone()
    B.tabx_layer_norm_backward(x, w, mean, rstd, alone, alone, row_mask=on)
    assert torch.equal(alone, want)
