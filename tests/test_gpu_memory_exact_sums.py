"""Linear attention of whole numbers so small that every sum of 32 bits is exact, in any order: what comes out has to be the
exact value, rounded once to its type.  Of bf16 arrays the products of queries and keys and the state that is read may be
off by 2^-17 of themselves."""
import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SPLIT = 2.0 ** -17             # two parts of eight bits, each to nearest: 2^-8 of a value, then 2^-9 of what is left at most
R, H, T = 2, 2, 40             # (a chunk of 32 ticks and a part of one; or a part of one of 64)
SCALE = 2.0 ** -9              # sums of 2^24 fit f16


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def whole(g, low, high, *shape):
    return torch.randint(low, high + 1, shape, generator=g).double()


def reach(K, dtype):
    """Up to where vectors of K whole numbers go whose products have some 19 bits and a sign (of bf16 elements: as many as
    their eight bits allow)."""
    return min(256 if dtype is BF16 else 2047, int((3.0 * 2.0 ** 19 / K ** 0.5) ** 0.5))


TAKEN = [3, 4, 35, 36]         # ticks that take something in: sums of four such products have less than 24 bits


def at_times(x):
    """x at those ticks; nothing at others."""
    out = torch.zeros_like(x)
    out[TAKEN] = x[TAKEN]
    return out


def exact(x, y, z, s0, order):
    """x_t S_t for t in order, S taking y z^T in before; and the sum of the magnitudes of what an implementation may round:
    products of x and y times z, elements of x times the state's (at any tick).  All below 2^24, so that 32 bits hold every
    sum of them in any order."""
    S = torch.zeros(R, H, x.shape[-1], z.shape[-1], dtype=torch.float64) if s0 is None else s0.clone()
    out, most = torch.zeros(T, R, H, z.shape[-1], dtype=torch.float64), S.abs()
    for t in order:
        S = S + y[t][..., :, None] * z[t][..., None, :]
        out[t] = (x[t][..., :, None] * S).sum(-2)
        most = torch.maximum(most, S.abs())
    scores = torch.einsum("trhk,srhk->trhs", x, y)
    magnitude = torch.einsum("trhs,srhv->trhv", scores.abs(), z.abs()) + torch.einsum("trhk,rhkv->trhv", x.abs(), most)
    assert magnitude.max() < 2 ** 24 and torch.einsum("trhk,srhk->trhs", x.abs(), y.abs()).max() < 2 ** 24
    return out, magnitude, S


def check(got, value, magnitude, dtype, what):
    value = SCALE * value
    bound = SPLIT * SCALE * magnitude if dtype is BF16 else torch.zeros_like(value)
    if dtype is BF16:
        M.near(got, value, M.rounded(bound, value, BF16), what)
    else:
        assert torch.equal(got.cpu(), value.to(dtype)), what


def call(B, d, dtype, state):
    up = [x.to(dtype).cuda() for x in d]
    K, V = d[0].shape[-1], d[2].shape[-1]
    decay, out = torch.zeros(H, device="cuda"), torch.empty(T, R, H, V, dtype=dtype, device="cuda")
    after = torch.empty(R, H, K, V, device="cuda")
    s0 = None if state is None else state.float().cuda()
    ws = torch.empty(B.tabx_linear_attention_workspace(T, R, H, K, V), dtype=torch.uint8, device="cuda")
    B.tabx_linear_attention(*up[:3], decay, SCALE, out, None, s0, after, ws)
    grads = [torch.empty_like(x) for x in up[:3]]
    B.tabx_linear_attention_backward(*up[:3], decay, SCALE, up[3], *grads, None, s0, None, None, ws)
    one, steps = torch.zeros_like(after) if s0 is None else s0.clone(), torch.empty_like(out)
    for t in range(T):
        B.tabx_linear_attention_step(up[0][t], up[1][t], up[2][t], decay, SCALE, one, steps[t])
    return out, after, grads, steps, one


WIDTHS = [(16, 16), (32, 24), (64, 64), (40, 64), (96, 96), (70, 96), (128, 128), (128, 100)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("K,V", WIDTHS)
def test_products_of_queries_and_keys(B, K, V, dtype):
    """They nearly cancel: a tick's value is the one before's with the other sign, its key nearly the one before's."""
    g = torch.Generator().manual_seed(K + V)
    a = reach(K, dtype)
    q, k = whole(g, -a, a, T, R, H, K), whole(g, -a + 1, a - 1, T, R, H, K)
    v = at_times(2.0 * whole(g, 0, 1, T, R, H, V) - 1.0)
    for t in (3, 35):
        k[t + 1] = k[t] + whole(g, 0, 1, R, H, K) * (whole(g, 0, 3, R, H, K) == 0)
        v[t + 1] = -v[t]
    go = at_times(whole(g, -1, 1, T, R, H, V))
    value, magnitude, last = exact(q, k, v, None, range(T))
    assert dtype is BF16 or (torch.einsum("trhk,srhk->trhs", q, k[TAKEN]).abs() > 2 ** 19).any()
    out, after, grads, steps, one = call(B, (q, k, v, go), dtype, None)
    check(out, value, magnitude, dtype, "at once")
    assert torch.equal(steps.cpu(), (SCALE * value).to(dtype)), "one by one"
    assert torch.equal(after.cpu(), last.float()) and torch.equal(one.cpu(), last.float())
    value, magnitude, _ = exact(k, q, go, None, range(T - 1, -1, -1))
    check(grads[2], value, magnitude, dtype, "grad_v")


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("K,V", WIDTHS)
def test_products_of_values_and_their_gradients(B, K, V, dtype):
    g = torch.Generator().manual_seed(2 * K + V)
    a = reach(V, dtype)
    v, go = whole(g, -a, a, T, R, H, V), whole(g, -a, a, T, R, H, V)
    q, k = at_times(whole(g, -1, 1, T, R, H, K)), at_times(whole(g, -1, 1, T, R, H, K))
    _, _, grads, _, _ = call(B, (q, k, v, go), dtype, None)
    assert dtype is BF16 or (torch.einsum("trhk,srhk->trhs", v, go).abs() > 2 ** 19).any()
    check(grads[0], *exact(go, v, k, None, range(T))[:2], dtype, "grad_q")
    check(grads[1], *exact(v, go, q, None, range(T - 1, -1, -1))[:2], dtype, "grad_k")


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("K,V", WIDTHS)
def test_the_state_that_is_read(B, K, V, dtype):
    """A state of 20 bits, read by queries that take neighbours from each other."""
    g = torch.Generator().manual_seed(3 * K + V)
    s0 = whole(g, -2 ** 19, 2 ** 19, R, H, K, V)
    s0[:, :, 1::2] = s0[:, :, 0::2] + whole(g, -8, 8, R, H, K // 2, V)
    q = torch.zeros(T, R, H, K, dtype=torch.float64)
    q[..., 4:16:2] = whole(g, -1, 1, T, R, H, 6)
    q[..., 5:16:2] = -q[..., 4:16:2]
    k, v, go = (whole(g, -1, 1, T, R, H, n) for n in (K, V, V))
    go[..., 9:] = 0.0
    value, magnitude, last = exact(q, k, v, s0, range(T))
    out, after, grads, steps, one = call(B, (q, k, v, go), dtype, s0)
    check(out, value, magnitude, dtype, "at once")
    assert torch.equal(steps.cpu(), (SCALE * value).to(dtype)), "one by one"
    assert torch.equal(after.cpu(), last.float()) and torch.equal(one.cpu(), last.float())
    value, magnitude, _ = exact(go, v, k, s0.transpose(-1, -2), range(T))
    check(grads[0], value, magnitude, dtype, "grad_q")
