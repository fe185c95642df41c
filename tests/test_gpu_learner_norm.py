"""Layer norm of rows and its gradients against 64-bit formulas (needs an MI355X)."""
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


def _say(*a):
    print("[gpu]", *a, flush=True)


def _rows(rng, rows, width, pad, dtype, scale=1.0, shift=0.0, offset=0):
    """A [rows, width] view whose rows lie width + pad apart, `offset` elements into its storage,
    amid values nobody may touch."""
    whole = torch.full((offset + rows * (width + pad),), 7.0, dtype=dtype, device=DEV)
    view = whole[offset:].view(rows, width + pad)[:, :width]
    view.copy_(torch.from_numpy(rng.normal(size=(rows, width)) * scale + shift))
    return whole, view


def _mask(rng, rows, share):
    return None if share is None else torch.from_numpy((rng.random(rows) < share).astype(np.uint8)).to(DEV)


def _outside(whole, view, want=7.0):
    """Nothing between the rows has been written."""
    left = torch.ones_like(whole, dtype=torch.bool)
    left.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    assert bool((whole[left] == want).all())


# (rows, width, pad of x, pad of y, type of x, type of y, share of rows that count, offset)
FORWARD = [
    (1, 1, 0, 0, F32, F32, None, 0), (3, 2, 0, 1, F32, BF16, None, 1), (7, 3, 2, 0, BF16, F32, 0.5, 1),
    (96, 96, 0, 0, F32, F32, None, 0), (65, 5, 0, 0, F16, F16, 0.3, 3), (33, 31, 1, 0, F32, F16, 0.5, 0),
    (257, 32, 0, 0, BF16, BF16, None, 0), (64, 33, 0, 3, F32, F32, 0.9, 1), (31, 64, 0, 0, F32, BF16, 0.0, 0),
    (100, 65, 0, 0, BF16, BF16, 0.5, 1), (77, 127, 1, 1, F16, F32, None, 0), (50, 128, 0, 0, F32, F32, 0.5, 2),
    (41, 129, 0, 0, F32, F32, None, 1), (129, 192, 0, 0, F32, BF16, 0.5, 0), (20, 255, 0, 5, F16, BF16, None, 0),
    (37, 256, 0, 0, BF16, F16, 0.4, 0), (340, 314, 0, 0, F32, F32, 0.5, 0), (60, 368, 0, 0, F32, BF16, 0.5, 0),
    (23, 384, 16, 0, BF16, BF16, None, 5), (19, 511, 0, 1, F32, F32, 0.5, 1), (18, 512, 0, 0, BF16, BF16, None, 0),
    (17, 513, 0, 0, F32, BF16, 0.6, 0), (9, 770, 2, 2, F16, F16, None, 1), (11, 1024, 0, 0, F32, BF16, None, 0),
    (10, 1025, 0, 0, F32, F32, 0.5, 1), (9, 2047, 0, 0, BF16, BF16, None, 0), (12, 2048, 0, 0, F32, BF16, 0.5, 0),
    (7, 2144, 0, 0, F32, F32, None, 0), (6, 2900, 4, 0, F32, F16, 0.5, 0), (5, 4096, 0, 0, F32, F32, None, 0),
    (5, 4097, 0, 0, BF16, F32, 0.5, 1), (4, 8192, 0, 0, F32, BF16, None, 0), (3, 6001, 0, 0, F16, F16, None, 0),
    (3, 7289, 1, 0, F32, F32, 0.7, 0), (5, 8192, 0, 0, BF16, BF16, 0.5, 0), (2, 8191, 0, 0, F32, F32, None, 3),
    # the narrowest and widest rows of every form that the others leave out
    (70, 4, 0, 0, F32, BF16, 0.5, 0), (70, 4, 1, 3, BF16, F16, None, 1), (900, 1, 0, 0, F16, F32, 0.5, 0),
    (35, 66, 0, 0, F32, F32, 0.5, 1), (35, 63, 3, 0, F16, F32, None, 0), (29, 130, 0, 0, BF16, BF16, 0.5, 0),
    (13, 257, 0, 0, F32, BF16, None, 1), (13, 259, 0, 0, F16, F16, 0.5, 0), (13, 516, 0, 0, F32, F32, None, 0),
    (300, 8, 0, 0, F32, F32, 0.5, 0), (301, 16, 0, 0, BF16, BF16, None, 0), (90, 17, 0, 0, F32, BF16, 0.5, 1),
    (500, 14, 3, 1, F16, F32, 0.5, 0), (200, 30, 0, 0, F32, F32, 0.5, 0), (77, 36, 0, 0, BF16, F32, None, 0),
    (13, 768, 0, 0, BF16, BF16, 0.5, 0), (13, 769, 1, 0, F32, F32, None, 1), (7, 2049, 0, 1, F32, F32, 0.5, 0),
    (7, 3070, 0, 0, BF16, BF16, None, 1), (7, 3073, 0, 0, F32, F16, 0.5, 0), (5, 4098, 2, 0, F16, BF16, None, 0),
]


@pytest.mark.parametrize("rows,width,px,py,tx,ty,share,offset", FORWARD)
def test_forward(B, rows, width, px, py, tx, ty, share, offset):
    _say("norm", rows, width, px, py, tx, ty, share, offset)
    rng = np.random.default_rng(rows * 1000 + width)
    wx, x = _rows(rng, rows, width, px, tx, 3.0, 1.5, offset)
    wy, y = _rows(rng, rows, width, py, ty, offset=offset)
    weight = torch.from_numpy(rng.normal(size=width) + 1).float().to(DEV)
    bias = torch.from_numpy(rng.normal(size=width)).float().to(DEV)
    mask = _mask(rng, rows, share)
    mean, rstd = torch.full((rows,), 9.0, device=DEV), torch.full((rows,), 9.0, device=DEV)
    before_x, before_y = wx.clone(), y.clone()
    B.tabx_layer_norm(x, weight, bias, 1e-5, y, mean, rstd, mask)
    torch.cuda.synchronize()
    wy_, wm, wr, by, bm, br = R.norm(R.f64(x), R.f64(weight), R.f64(bias), float(np.float32(1e-5)), ty)
    on = np.ones(rows, bool) if mask is None else mask.cpu().numpy() != 0
    R.near(R.f64(y)[on], wy_[on], by[on], "y")
    R.near(R.f64(mean)[on], wm[on], bm[on], "mean")
    R.near(R.f64(rstd)[on], wr[on], br[on], "rstd")
    off = torch.from_numpy(~on).to(DEV)
    assert torch.equal(y[off], before_y[off])
    assert bool((mean[off] == 9).all()) and bool((rstd[off] == 9).all())
    assert torch.equal(wx, before_x)
    _outside(wy, y)


def test_forward_without_weight_bias_or_statistics(B):
    rng = np.random.default_rng(1)
    _, x = _rows(rng, 40, 100, 0, F32)
    for w, b in ((None, None), (torch.full((100,), 2.0, device=DEV), None), (None, torch.ones(100, device=DEV))):
        y = torch.empty(40, 100, device=DEV)
        B.tabx_layer_norm(x, w, b, 1e-6, y)
        want, _, _, bound, _, _ = R.norm(R.f64(x), None if w is None else R.f64(w), None if b is None else R.f64(b),
                                         float(np.float32(1e-6)), F32)
        R.near(y, want, bound, "y")


def test_rows_of_zeros_and_of_what_is_not_finite(B):
    """A disabled unit's row of zeros has the bias; infinity and NaN stay in their own rows, and in
    rows that are masked out nobody meets them."""
    rng = np.random.default_rng(2)
    _, x = _rows(rng, 64, 368, 0, F32)
    x[5] = 0.0
    x[9, 3], x[17, 100], x[40, 367] = float("inf"), float("nan"), float("-inf")
    bias = torch.from_numpy(rng.normal(size=368)).float().to(DEV)
    mask = torch.ones(64, dtype=torch.uint8, device=DEV)
    mask[17] = 0
    y = torch.full((64, 368), 3.0, device=DEV)
    mean, rstd = torch.zeros(64, device=DEV), torch.zeros(64, device=DEV)
    B.tabx_layer_norm(x, None, bias, 1e-5, y, mean, rstd, mask)
    assert torch.equal(y[5], bias) and bool((y[17] == 3).all())
    fine = torch.isfinite(y).all(1)
    assert not fine[9] and not fine[40] and int(fine.sum()) == 62
    gy = torch.from_numpy(rng.normal(size=(64, 368))).float().to(DEV)
    gy[9], gy[40] = 1.0, 1.0
    mask[9] = mask[40] = 0
    gx = torch.empty(64, 368, device=DEV)
    gw, gb = torch.empty(368, device=DEV), torch.empty(368, device=DEV)
    ws = torch.empty(B.tabx_layer_norm_workspace(64, 368), dtype=torch.uint8, device=DEV)
    B.tabx_layer_norm_backward(x, None, mean, rstd, gy, gx, gw, gb, ws, mask)
    assert bool(torch.isfinite(gx).all()) and bool(torch.isfinite(gw).all()) and bool(torch.isfinite(gb).all())
    assert bool((gx[[9, 17, 40]] == 0).all())


def test_in_place(B):
    rng = np.random.default_rng(3)
    for width in (96, 368, 1030, 5000):
        _, x = _rows(rng, 30, width, 3, F32)
        want = torch.empty(30, width, device=DEV)
        B.tabx_layer_norm(x, None, None, 1e-5, want)
        B.tabx_layer_norm(x, None, None, 1e-5, x)
        assert torch.equal(x, want)


def _turns(B, rows, width):
    """Rows one lane adds up, at most: those of its workgroup, of which a workgroup of rows of up to 1024
    elements has at least four side by side."""
    groups = B.tabx_layer_norm_workspace(rows, width) // (8 * width)
    return -(-rows // groups) + 64


# (rows, width, pad, type of x, type of the gradients, share, input's gradient, weight's, bias's)
BACKWARD = [
    (1, 1, 0, F32, F32, None, True, True, True), (5, 2, 1, F32, BF16, None, False, True, True),
    (300, 3, 0, BF16, BF16, 0.5, True, True, True), (96, 96, 0, F32, F32, None, True, True, True),
    (513, 33, 3, F16, F16, 0.5, True, True, True), (1000, 64, 0, F32, BF16, None, False, True, True),
    (130, 100, 0, BF16, F32, 0.7, True, True, False), (129, 128, 0, F32, F32, None, True, False, True),
    (77, 130, 1, F32, F32, 0.5, True, True, True), (2000, 192, 0, BF16, BF16, None, True, True, True),
    (260, 250, 0, F16, BF16, 0.0, True, True, True), (700, 256, 0, F32, F32, 0.5, False, True, True),
    (5003, 314, 0, F32, F32, 0.5, True, True, True), (4099, 368, 0, F32, BF16, 0.5, False, True, True),
    (1025, 384, 0, BF16, BF16, None, True, True, True), (999, 512, 0, BF16, BF16, None, True, True, True),
    (301, 515, 2, F32, F32, 0.5, True, True, True), (411, 768, 0, BF16, BF16, None, True, True, True),
    (203, 1000, 0, F16, F16, None, True, True, True), (333, 1024, 0, BF16, BF16, 0.5, True, False, False),
    (65, 1500, 0, F32, BF16, None, False, True, True), (57, 2048, 0, F32, BF16, None, True, True, True),
    (33, 2144, 0, F32, F32, 0.5, True, True, True), (21, 4001, 1, BF16, BF16, None, True, True, True),
    (14, 4100, 0, F32, F32, None, True, True, True), (9, 8192, 0, BF16, BF16, 0.5, True, True, True),
    (5, 7001, 0, F32, F32, None, False, True, True), (7, 8192, 0, F16, F16, None, True, True, True),
    (4, 8191, 3, F32, F32, 0.5, True, True, True), (300, 4, 0, F32, BF16, 0.5, True, True, True),
    (77, 4, 1, BF16, F32, None, False, True, True), (3000, 16, 0, F32, F32, 0.5, True, True, True),
    (2001, 13, 1, BF16, BF16, 0.5, True, True, True), (900, 32, 0, F32, BF16, None, False, True, True),
    (700, 18, 0, F16, F32, 0.5, True, True, False), (70, 66, 0, F32, F32, 0.5, True, True, True),
    (70, 131, 0, F16, F16, None, True, True, True), (30, 257, 1, F32, BF16, 0.5, True, True, True),
    (30, 260, 0, BF16, BF16, None, False, True, True), (30, 769, 0, F32, F32, 0.5, True, True, True),
    (9, 1026, 0, BF16, F32, None, True, True, True), (9, 2049, 0, F32, F32, 0.5, False, True, True),
    (9, 2050, 0, F16, F16, None, True, True, True), (9, 3074, 3, F32, BF16, None, True, True, True),
    (9, 4099, 0, F32, F32, 0.5, True, True, True),
]


@pytest.mark.parametrize("rows,width,pad,tx,tg,share,inputs,weights,biases", BACKWARD)
def test_backward(B, rows, width, pad, tx, tg, share, inputs, weights, biases):
    _say("norm grad", rows, width, pad, tx, tg, share, inputs, weights, biases)
    rng = np.random.default_rng(rows * 1000 + width)
    _, x = _rows(rng, rows, width, pad, tx, 3.0, 1.5, 1)
    _, gy = _rows(rng, rows, width, pad, tg)
    whole, gx = _rows(rng, rows, width, pad, tx)
    weight = torch.from_numpy(rng.normal(size=width) + 1).float().to(DEV) if width % 2 else None
    mean = x.float().mean(1).contiguous()
    rstd = torch.rsqrt(x.float().var(1, unbiased=False) + 1e-5).contiguous()
    mask = _mask(rng, rows, share)
    gw = torch.full((width,), 5.0, device=DEV) if weights else None
    gb = torch.full((width,), 5.0, device=DEV) if biases else None
    size = B.tabx_layer_norm_workspace(rows, width)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device=DEV)       # its contents need no preparation
    B.tabx_layer_norm_backward(x, weight, mean, rstd, gy, gx if inputs else None, gw, gb, ws[:size], mask)
    on = np.ones(rows, bool) if mask is None else mask.cpu().numpy() != 0
    wx, ww, wb, bx, bw, bb = R.norm_grad(R.f64(x), on, None if weight is None else R.f64(weight), R.f64(mean), R.f64(rstd),
                                         R.f64(gy), tx, _turns(B, rows, width))
    if inputs:
        R.near(gx, wx, bx, "grad_x")
        _outside(whole, gx)
    if weights:
        R.near(gw, ww, bw, "grad_weight")
    if biases:
        R.near(gb, wb, bb, "grad_bias")
    assert bool((ws[size:] == 255).all())
    # the same sums in the same order
    gw2, gb2 = (None if t is None else torch.empty_like(t) for t in (gw, gb))
    B.tabx_layer_norm_backward(x, weight, mean, rstd, gy, None if (weights or biases) else gx, gw2, gb2, ws[:size], mask)
    assert gw is None or torch.equal(gw, gw2)
    assert gb is None or torch.equal(gb, gb2)


@pytest.mark.parametrize("width", [1, 3, 4, 18, 33, 96, 130, 314, 515, 1026, 2048, 4099, 8191])
@pytest.mark.parametrize("rows", [1, 4, 8, 9])
def test_weight_gradients_of_few_rows(B, rows, width):
    """Each of the two alone and both, with nothing written around them, in a first and in a second call."""
    _say("norm grad of few rows", rows, width)
    rng = np.random.default_rng(rows * 10000 + width)
    _, x = _rows(rng, rows, width, 1, F32, 2.0, 1.0, 1)
    _, gy = _rows(rng, rows, width, 0, F32)
    mean = x.mean(1).contiguous()
    rstd = torch.rsqrt(x.var(1, unbiased=False) + 1e-5).contiguous()
    _, ww, wb, _, bw, bb = R.norm_grad(R.f64(x), np.ones(rows, bool), None, R.f64(mean), R.f64(rstd), R.f64(gy), F32, rows + 64)
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    for weights, biases in ((True, True), (True, False), (False, True)):
        whole = torch.full((2, width + 16), 7.0, device=DEV)
        gw, gb = (whole[i, 8:8 + width] if on else None for i, on in enumerate((weights, biases)))
        for _ in range(2):
            B.tabx_layer_norm_backward(x, None, mean, rstd, gy, None, gw, gb, ws)
        if weights:
            R.near(gw, ww, bw, "grad_weight")
        if biases:
            R.near(gb, wb, bb, "grad_bias")
        for i, on in enumerate((weights, biases)):
            assert bool((whole[i, :8] == 7).all()) and bool((whole[i, 8 + width:] == 7).all())
            assert on or bool((whole[i] == 7).all())


def test_gradient_against_differences(B):
    """sum(gy * norm(x)) along random directions, from the forward call in float32: a central
    difference of step h is off by h^2 and by the rounding of two sums over h."""
    rng = np.random.default_rng(7)
    rows, width = 50, 90
    x = torch.from_numpy(rng.normal(size=(rows, width))).float().to(DEV)
    w = torch.from_numpy(rng.normal(size=width) + 1).float().to(DEV)
    b = torch.from_numpy(rng.normal(size=width)).float().to(DEV)
    gy = torch.from_numpy(rng.normal(size=(rows, width))).float().to(DEV)
    mean, rstd, y = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(x)

    def loss(x_, w_, b_):
        out = torch.empty_like(x_)
        B.tabx_layer_norm(x_, w_, b_, 1e-5, out)
        return float((out.double() * gy.double()).sum())

    B.tabx_layer_norm(x, w, b, 1e-5, y, mean, rstd)
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    B.tabx_layer_norm_backward(x, w, mean, rstd, gy, gx, gw, gb, ws)
    h = 2.0 ** -8
    for t, g, at in ((x, gx, 0), (w, gw, 1), (b, gb, 2)):
        d = torch.from_numpy(rng.normal(size=tuple(t.shape))).float().to(DEV)
        args = [x, w, b]
        up, down = list(args), list(args)
        up[at], down[at] = t + h * d, t - h * d
        slope = (loss(*up) - loss(*down)) / (2 * h)
        want = float((g.double() * d.double()).sum())
        # third derivatives of a normalised row times a unit direction are of the order of the
        # gradient's own magnitude; 4500 roundings of half a step add as a random walk
        scale = float((g.double().abs() * d.double().abs()).sum())
        rounding = 8 * 2.0 ** -24 * float((y.double().abs() * gy.double().abs()).sum()) / h
        assert abs(slope - want) <= 8 * h * h * scale + rounding, (at, slope, want)


def test_gradients_in_place_and_far_rows(B):
    """grad_x may be grad_y; rows whose offsets pass 32 bits (4.3e9 elements apart in all)."""
    rng = np.random.default_rng(8)
    for width in (100, 700, 3000):
        x = torch.from_numpy(rng.normal(size=(20, width))).float().to(DEV)
        gy = torch.from_numpy(rng.normal(size=(20, width))).float().to(DEV)
        mean, rstd = x.mean(1), torch.rsqrt(x.var(1, unbiased=False) + 1e-5)
        gx = torch.empty_like(x)
        B.tabx_layer_norm_backward(x, None, mean, rstd, gy, gx)
        B.tabx_layer_norm_backward(x, None, mean, rstd, gy, gy)
        assert torch.equal(gx, gy)
    stride, rows, width = 1 << 21, 2050, 40
    x = torch.empty(rows * stride, dtype=BF16, device=DEV).view(rows, stride)[:, :width]
    x.copy_(torch.from_numpy(rng.normal(size=(rows, width))))
    y, near = torch.empty(rows, width, device=DEV), torch.empty(rows, width, device=DEV)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    B.tabx_layer_norm(x.contiguous(), None, None, 1e-5, near)
    B.tabx_layer_norm(x, None, None, 1e-5, y, mean, rstd)
    assert torch.equal(y, near)
    gy = torch.from_numpy(rng.normal(size=(rows, width))).float().to(DEV)
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    got = []
    for rows_of in (x, x.contiguous()):
        gx, gw, gb = torch.empty(rows, width, device=DEV), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
        B.tabx_layer_norm_backward(rows_of, None, mean, rstd, gy, gx, gw, gb, ws)
        got.append((gx, gw, gb))
    for p, q in zip(*got):
        assert torch.equal(p, q)


def test_no_rows(B):
    e = torch.empty(0, 64, device=DEV)
    r = torch.empty(0, device=DEV)
    B.tabx_layer_norm(e, None, None, 1e-5, e.clone(), r, r.clone())
    gw = torch.ones(64, device=DEV)
    ws = torch.empty(B.tabx_layer_norm_workspace(0, 64), dtype=torch.uint8, device=DEV)
    B.tabx_layer_norm_backward(e, None, r, r, e, None, gw, gw.clone(), ws)
    torch.cuda.synchronize()
    assert bool((gw == 0).all())                                # a sum over no rows
