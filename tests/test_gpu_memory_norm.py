"""Root-mean-square norm behind a residual addition, to 8 bits too, and its gradients, against 64 bits."""
import math

import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
F32, BF16, F16, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
EPS = 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def rows(g, R, W, dtype, size=1.0, pad=0):
    wide = (size * torch.randn(R, W + pad, generator=g)).to(dtype)
    return wide[:, :W]


def run(B, x, residual, weight, sum_type, out_type, mask=None, wanted=True):
    R, W = x.shape
    s = None if sum_type is None else torch.full((R, W), 7.0, dtype=sum_type, device="cuda")
    y = torch.full((R, W), 7.0, device="cuda").to(out_type)
    scale = torch.full((R,), 7.0, device="cuda") if out_type is E4M3 else None
    rstd = torch.full((R,), 7.0, device="cuda") if wanted else None
    up = [None if t is None else t.cuda() for t in (x, residual, weight, mask)]
    B.tabx_rms_norm(up[0], up[2], EPS, y, scale, rstd, up[1], s, up[3])
    got = {"sum": s, "y": y, "scale": scale, "rstd": rstd}
    return {n: t for n, t in got.items() if t is not None}


WIDTHS = [1, 2, 3, 4, 5, 15, 16, 17, 32, 33, 63, 64, 65, 96, 128, 130, 192, 193, 256, 260, 384, 511, 512, 700, 768, 769, 1000, 1024,
          1030, 1536, 1537, 2048, 2050, 4095, 4097, 6000, 8192]


@pytest.mark.parametrize("W", WIDTHS)
def test_every_form(B, W):
    g = torch.Generator().manual_seed(W)
    for types in ((F32, None, None, F32), (BF16, BF16, BF16, BF16), (BF16, F32, F32, E4M3), (F16, F16, None, F16), (F32, BF16, BF16, E4M3),
                  (F16, None, F16, BF16)):
        xt, rt, st, yt = types
        R = 37
        x = rows(g, R, W, xt, pad=W % 3)
        residual = None if rt is None else rows(g, R, W, rt, 3.0, pad=W % 2)
        weight = None if W % 5 == 0 else 1.0 + torch.randn(W, generator=g)
        for n, t in run(B, x, residual, weight, st, yt).items():
            M.near(t, *M.norm(x, residual, weight, EPS, st, yt)[n], (W, types, n))


@pytest.mark.parametrize("W", [3, 40, 130, 1000, 4097])
def test_rows_left_out_stay(B, W):
    g = torch.Generator().manual_seed(1)
    x, residual = rows(g, 300, W, BF16), rows(g, 300, W, BF16)
    mask = (torch.rand(300, generator=g) < 0.5).to(torch.uint8)
    mask[64:140] = 0
    off = mask == 0
    x[off], residual[off] = math.nan, math.nan
    for yt in (BF16, E4M3):
        got = run(B, x, residual, None, BF16, yt, mask)
        want = M.norm(x, residual, None, EPS, BF16, yt)
        for n, t in got.items():
            on = mask != 0
            M.near(t.float().cpu()[on], want[n][0][on], want[n][1][on], n)
            assert (t.float().cpu()[off] == 7.0).all(), n


def test_in_place(B):
    g = torch.Generator().manual_seed(2)
    for W in (20, 96, 512, 1000, 2500):
        x, residual = rows(g, 500, W, F32), rows(g, 500, W, F32)
        want = M.norm(x, residual, None, EPS, F32, F32)
        for sum_is in ("x", "residual"):
            a, b, y = x.cuda(), residual.cuda(), torch.empty(500, W, device="cuda")
            s = a if sum_is == "x" else b
            B.tabx_rms_norm(a, None, EPS, y, None, None, b, s)
            M.near(s, *want["sum"], sum_is)
            M.near(y, *want["y"], sum_is)
            a, b, s = x.cuda(), residual.cuda(), torch.empty(500, W, device="cuda")
            y = a if sum_is == "x" else b
            B.tabx_rms_norm(a, None, EPS, y, None, None, b, s)
            M.near(y, *want["y"], sum_is)
            M.near(s, *want["sum"], sum_is)


def test_eight_bits_at_their_ends(B):
    """Rows of zeros, of the smallest and the largest values, of one large value, not finite ones."""
    W = 70
    x = torch.zeros(8, W)
    x[1] = 1e-38
    x[2] = 1e18
    x[3, 5] = 1.0
    x[4] = torch.linspace(-1, 1, W)
    x[5, 3] = math.nan
    x[6, 3] = math.inf
    x[7] = torch.logspace(-12, 0, W)
    weight = torch.ones(W)
    got = run(B, x, None, weight, None, E4M3)
    want = M.norm(x[:5], None, weight, EPS, None, E4M3)
    for n in ("y", "scale", "rstd"):
        M.near(got[n][:5].float(), want[n][0], want[n][1], n)
    y = got["y"].float().cpu()
    assert (y[0] == 0).all() and got["scale"][0] == 2.0 ** -126
    assert y[4].abs().max() == 448.0 and y[3, 5] == 448.0
    # of a row with a value that is no number none is one; beside an infinite one there are zeros
    assert torch.isnan(y[5]).all() and torch.isnan(y[6, 3]) and (y[6, :3] == 0).all() and (y[6, 4:] == 0).all()
    last = M.norm(x[7:], None, weight, EPS, None, E4M3)
    M.near(got["y"][7:].float(), *last["y"], "small ones")


def test_scaled_rows_stand_for_the_norm(B):
    """What a product in 8 bits multiplies out: y times scale is the norm to four bits."""
    g = torch.Generator().manual_seed(3)
    x = rows(g, 64, 512, BF16)
    got = run(B, x, None, None, None, E4M3)
    whole = M.norm(x, None, None, EPS, None, F32)["y"][0]
    back = got["y"].double().cpu() * got["scale"].double().cpu()[:, None]
    most = whole.abs().amax(1, keepdim=True)
    assert ((back - whole).abs() <= 2.0 ** -4 * whole.abs() + most / 448 * 2.0 ** -10 + 1e-5 * most).all()


TURNS = 4000                   # rows that one lane adds up here, at most


@pytest.mark.parametrize("W", WIDTHS)
def test_gradients(B, W):
    g = torch.Generator().manual_seed(W)
    for xt, gt, ot, stream, R in ((F32, F32, F32, True, 37), (BF16, BF16, BF16, True, 500), (BF16, F32, F32, False, 131), (F32, F16, BF16, False, 1),
                                  (F16, F16, F16, True, 90)):
        s, gy = rows(g, R, W, xt, 2.0, pad=W % 3), rows(g, R, W, gt, pad=W % 2)
        gs = rows(g, R, W, xt) if stream else None
        weight = None if W % 5 == 0 else 1.0 + torch.randn(W, generator=g)
        mask = None if R < 100 else (torch.rand(R, generator=g) < 0.6).to(torch.uint8)
        on = torch.ones(R, dtype=torch.bool) if mask is None else mask != 0
        if mask is not None:
            s[~on], gy[~on] = math.nan, math.nan
        rstd = torch.rsqrt((s.float() ** 2).mean(1) + EPS)
        gx, gw = torch.full((R, W), 7.0, dtype=ot, device="cuda"), torch.full((W,), 7.0, device="cuda")
        ws = torch.empty(B.tabx_rms_norm_workspace(R, W), dtype=torch.uint8, device="cuda")
        up = [None if t is None else t.cuda() for t in (s, weight, rstd, gy, gs, mask)]
        B.tabx_rms_norm_backward(up[0], up[1], up[2], up[3], up[4], gx, gw, ws, up[5])
        clean = [torch.nan_to_num(t) if t is not None else None for t in (s, gy, gs)]
        want = M.norm_grad(clean[0], weight, torch.nan_to_num(rstd), clean[1], clean[2], on, ot, TURNS)
        M.near(gx, *want["grad_x"], (W, xt))
        M.near(gw, *want["grad_weight"], (W, xt))
        alone = torch.full((W,), 7.0, device="cuda")
        B.tabx_rms_norm_backward(up[0], up[1], up[2], up[3], up[4], None, alone, ws, up[5])
        M.near(alone, *want["grad_weight"], (W, xt))
        only = torch.full((R, W), 7.0, dtype=ot, device="cuda")
        B.tabx_rms_norm_backward(up[0], up[1], up[2], up[3], up[4], only, None, None, up[5])
        assert torch.equal(only, gx)


def test_gradient_in_place_and_of_no_rows(B):
    g = torch.Generator().manual_seed(5)
    for W in (40, 512, 1500):
        s, gy, gs = (rows(g, 300, W, F32) for _ in range(3))
        rstd = torch.rsqrt((s ** 2).mean(1) + EPS)
        want = M.norm_grad(s, None, rstd, gy, gs, torch.ones(300, dtype=torch.bool), F32, TURNS)
        for which in (0, 1):
            a, b = gy.cuda(), gs.cuda()
            B.tabx_rms_norm_backward(s.cuda(), None, rstd.cuda(), a, b, (a, b)[which])
            M.near((a, b)[which], *want["grad_x"], which)
    none, gw = torch.zeros(0, 40, device="cuda"), torch.full((40,), 7.0, device="cuda")
    ws = torch.empty(B.tabx_rms_norm_workspace(0, 40), dtype=torch.uint8, device="cuda")
    B.tabx_rms_norm_backward(none, None, none[:, 0].contiguous(), none, None, none.clone(), gw, ws)
    assert (gw == 0).all()
    B.tabx_rms_norm(none, None, EPS, none.clone())


def test_gradients_against_differences():
    """The formula is the slope of the norm's: autograd's of the definition, in 64 bits."""
    g = torch.Generator().manual_seed(6)
    x = torch.randn(5, 7, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(7, generator=g, dtype=torch.float64, requires_grad=True)
    gy, gs = (torch.randn(5, 7, generator=g, dtype=torch.float64) for _ in range(2))
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    ((x * rstd * w * gy).sum() + (x * gs).sum()).backward()
    want = M.norm_grad(x, w, rstd[:, 0], gy, gs, torch.ones(5, dtype=torch.bool), F32, 1)
    assert torch.allclose(want["grad_x"][0], x.grad, rtol=0, atol=1e-12)
    assert torch.allclose(want["grad_weight"][0], w.grad, rtol=0, atol=1e-12)


def test_large_calls_are_the_small_ones(B):
    """More rows than a launch has teams, results past the caches: bit for bit the same rows alone."""
    g = torch.Generator("cuda").manual_seed(7)
    for R, W in ((200001, 512), (1500007, 24), (20011, 2100)):
        x, residual = (torch.randn(R, W, generator=g, device="cuda").to(BF16) for _ in range(2))
        mask = (torch.rand(R, generator=g, device="cuda") < 0.7).to(torch.uint8)
        s, y = torch.full_like(x, 7.0), torch.full((R, W), 7.0, device="cuda").to(E4M3)
        scale, rstd = torch.full((R,), 7.0, device="cuda"), torch.full((R,), 7.0, device="cuda")
        B.tabx_rms_norm(x, None, EPS, y, scale, rstd, residual, s, mask)
        for at in (0, R // 2, R - 9):
            c = slice(at, at + 9)
            s1, y1 = torch.full_like(x[c], 7.0), torch.full((9, W), 7.0, device="cuda").to(E4M3)
            sc1, r1 = torch.full((9,), 7.0, device="cuda"), torch.full((9,), 7.0, device="cuda")
            B.tabx_rms_norm(x[c], None, EPS, y1, sc1, r1, residual[c], s1, mask[c])
            for a, b in ((s, s1), (y.view(torch.uint8), y1.view(torch.uint8)), (scale, sc1), (rstd, r1)):
                assert torch.equal(a[c], b)


@pytest.mark.parametrize("W", [1025, 1030, 1537, 2049, 2050, 3071, 4093, 4097, 8190])
def test_gradient_in_the_streams_place_of_wide_rows(B, W):
    """Rows that several wavefronts share: the last elements, which more than one of them reads, are read before they are
    overwritten; bit for bit what a call with an output of its own gives."""
    g = torch.Generator("cuda").manual_seed(W)
    R = 1500
    for t in (F32, BF16):
        s, gy, gs = (torch.randn(R, W, generator=g, device="cuda").to(t) for _ in range(3))
        rstd = torch.rsqrt((s.float() ** 2).mean(1) + EPS)
        apart, together = torch.full_like(s, 7.0), gs.clone()
        B.tabx_rms_norm_backward(s, None, rstd, gy, gs, apart)
        B.tabx_rms_norm_backward(s, None, rstd, gy, together, together)
        assert torch.equal(apart, together), t
        some = torch.arange(0, R, 97)
        want = M.norm_grad(s.cpu()[some], None, rstd.cpu()[some], gy.cpu()[some], gs.cpu()[some], torch.ones(len(some), dtype=torch.bool), t, 1)
        M.near(together.cpu()[some], *want["grad_x"], t)
