"""Rotation of pairs by several axes, against 64 bits."""
import math

import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def make(seed, R, H, W, pairs, dtype, units=1, far=1000):
    """x [R, H, W], axes of (t of each env, x, y, t of each unit) as many as `pairs` has, frequency."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, H, W, generator=g).to(dtype)
    places = [torch.randint(-far, far, (R // units,), generator=g).to(torch.int32), 64.0 * torch.rand(R, generator=g),
              -1000.0 + 2000.0 * torch.rand(R, generator=g), torch.randint(0, 10, (R,), generator=g).to(torch.int32)]
    frequency = torch.cat([100.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in pairs])
    return x, list(zip(places, pairs)), frequency


def run(B, x, axes, frequency, interleaved, inverse, mask=None, y=None):
    y = torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda") if y is None else y
    B.tabx_rotary(x.cuda(), [(p.cuda(), n) for p, n in axes], frequency.cuda(), y, interleaved, inverse,
                  None if mask is None else mask.cuda())
    return y


SHAPES = [(1, 1, 2, (1,)), (5, 3, 7, (3,)), (64, 2, 16, (3, 5)), (37, 4, 64, (10, 11, 11)), (20, 1, 65, (1, 0, 2, 5)),
          (300, 2, 40, (0, 15)), (9, 3, 128, (64,)), (12, 2, 250, (41, 42, 42)), (6, 2, 512, (64, 64, 64, 64)), (8, 20, 24, (4, 4, 4))]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_axes(B, shape, dtype):
    R, H, W, pairs = shape
    x, axes, frequency = make(1, R, H, W, pairs, dtype, units=2 if R % 2 == 0 else 1)
    for interleaved in (False, True):
        for inverse in (False, True):
            y = run(B, x, axes, frequency, interleaved, inverse)
            M.near(y, *M.rotary(x, axes, frequency, interleaved, inverse), (shape, dtype, interleaved, inverse))


@pytest.mark.parametrize("interleaved", [False, True])
def test_forth_and_back_in_place(B, interleaved):
    x, axes, frequency = make(2, 50, 3, 48, (7, 8, 8), torch.float32, units=5)
    y = x.cuda()
    B.tabx_rotary(y, [(p.cuda(), n) for p, n in axes], frequency.cuda(), y, interleaved)
    want, bound = M.rotary(x, axes, frequency, interleaved, False)
    M.near(y, want, bound, "in place")
    B.tabx_rotary(y, [(p.cuda(), n) for p, n in axes], frequency.cuda(), y, interleaved, True)
    # the way back of the bound, and its own: a rotation leaves lengths as they are
    M.near(y, x.double(), 2.0 * (bound + bound.roll(-1, -1) + bound.amax()), "and back")


def test_far_positions(B):
    """Angles of 2^31 radians: 64 bits keep what 32 would have lost."""
    x, _, _ = make(3, 40, 2, 8, (4,), torch.float32)
    position = torch.tensor([2 ** 31 - 1 - 7 * i for i in range(20)] + [-2 ** 31 + 3 * i for i in range(20)], dtype=torch.int64).to(torch.int32)
    frequency = torch.tensor([1.0, 0.1, 1e-3, math.pi], dtype=torch.float64)
    axes = [(position, 4)]
    M.near(run(B, x, axes, frequency, False, False), *M.rotary(x, axes, frequency, False, False), "far")


def test_quarters(B):
    """Angles at and around every eighth of a turn: which series, and which sign."""
    n = 64
    position = torch.cat([torch.full((1,), k * math.pi / 4) + d for k in range(-9, 10) for d in (torch.tensor([-1e-4]), torch.zeros(1), torch.tensor([1e-4]))])
    x = torch.randn(len(position), 1, 2, generator=torch.Generator().manual_seed(4))
    axes, frequency = [(position, 1)], torch.ones(1, dtype=torch.float64)
    M.near(run(B, x, axes, frequency, True, False), *M.rotary(x, axes, frequency, True, False), "quarters")
    assert n


def test_rows_left_out_and_positions_that_are_none(B):
    x, axes, frequency = make(5, 30, 2, 20, (4, 5), torch.bfloat16, units=3)
    mask = (torch.arange(30) % 3 != 1).to(torch.uint8)
    y = run(B, x, axes, frequency, False, False, mask)
    want, bound = M.rotary(x, axes, frequency, False, False)
    on = mask != 0
    M.near(y.cpu()[on], want[on], bound[on], "on")
    assert (y.cpu()[~on] == 7.0).all()
    axes[1][0][4] = math.inf
    y = M.f64(run(B, x, axes, frequency, False, False))
    turned = [i for i in range(9) if i >= 4] + [i + 9 for i in range(9) if i >= 4]
    rest = [i for i in range(20) if i not in turned]
    assert torch.isnan(y[4][:, turned]).all()
    M.near(y[4][:, rest], want[4][:, rest], bound[4][:, rest], "rest")
    keep = torch.arange(30) != 4
    M.near(y[keep], want[keep], bound[keep], "others")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_columns_of_a_projection(B, dtype):
    """Queries and keys side by side in rows of odd width, heads at distances of their own; what lies between stays."""
    R, H, W = 33, 5, 14
    x, axes, frequency = make(6, R, H, W, (3, 3), dtype)
    wide = torch.full((R, 3 + H * (W + 1) + 4), math.nan, dtype=dtype, device="cuda")
    view = wide[:, 3:3 + H * (W + 1)].unflatten(-1, (H, W + 1))[..., :W]
    view.copy_(x)
    y = wide.new_full((R, H, W + 6), 7.0)
    B.tabx_rotary(view, [(p.cuda(), n) for p, n in axes], frequency.cuda(), y[..., 2:2 + W])
    M.near(y[..., 2:2 + W], *M.rotary(x, axes, frequency, False, False), "columns")
    assert (y[..., :2] == 7.0).all() and (y[..., 2 + W:] == 7.0).all()
    B.tabx_rotary(view, [(p.cuda(), n) for p, n in axes], frequency.cuda(), view)
    M.near(view, *M.rotary(x, axes, frequency, False, False), "in place")


def test_many_rows(B):
    """More rows than a launch has lanes for at a time: the same bits as the last rows alone."""
    R, H, W = 9000007, 1, 8
    g = torch.Generator("cuda").manual_seed(7)
    x = torch.randn(R, H, W, generator=g, device="cuda").to(torch.bfloat16)
    t = torch.randint(0, 500, (R,), generator=g, device="cuda").to(torch.int32)
    frequency = torch.tensor([1.0, 0.3, 0.1, 0.03], dtype=torch.float64, device="cuda")
    y = torch.empty_like(x)
    B.tabx_rotary(x, [(t, 4)], frequency, y)
    for at in (0, R // 2, R - 11):
        c = slice(at, at + 11)
        z = torch.empty_like(x[c])
        B.tabx_rotary(x[c], [(t[c], 4)], frequency, z)
        assert torch.equal(y[c], z)


def test_more_rows_than_a_launch_has_workgroups(B):
    """Rows of which a workgroup takes one at a time, and some of them a second: the same bits as rows alone."""
    R, H, W = 2 ** 20 + 37, 1024, 2
    g = torch.Generator("cuda").manual_seed(8)
    x = torch.randn(1, H, W, generator=g, device="cuda").to(torch.bfloat16).expand(R, H, W)
    t = torch.randint(0, 500, (R,), generator=g, device="cuda").to(torch.int32)
    frequency = torch.tensor([0.7], dtype=torch.float64, device="cuda")
    y = torch.empty(R, H, W, dtype=torch.bfloat16, device="cuda")
    B.tabx_rotary(x, [(t, 1)], frequency, y)
    for at in (0, 2 ** 19, 2 ** 20 - 3, R - 5):
        c = slice(at, at + 5)
        z = torch.empty(5, H, W, dtype=torch.bfloat16, device="cuda")
        B.tabx_rotary(x[c], [(t[c], 1)], frequency, z)
        assert torch.equal(y[c], z), at
    M.near(z, *M.rotary(x[c].cpu(), [(t[c].cpu(), 1)], frequency.cpu(), False, False), "last ones")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rows_far_apart(B, dtype, interleaved):
    """Rows, and heads, whose distances pass 32 bits inside a workgroup."""
    R, H, W = 5, 3, 24
    x, axes, frequency = make(9, R, H, W, (4, 5), dtype)
    want = M.rotary(x, axes, frequency, interleaved, False)
    far = torch.empty(2 ** 32 + 2 ** 20, dtype=dtype, device="cuda")
    rows_far = far.as_strided((R, H, W), (2 ** 30 - 5, W + 1, 1), 7)
    heads_far = far.as_strided((R, H, W), (W + 3, 2 ** 31 - 3, 1), 2 ** 14)
    for view in (rows_far, heads_far):
        M.near(run(B, x, axes, frequency, interleaved, False, y=view), *want, "output")
        M.near(run(B, view, axes, frequency, interleaved, True), *M.rotary(view.cpu(), axes, frequency, interleaved, True), "input")
