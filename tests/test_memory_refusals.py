"""Which calls of a unit's memory are refused, on the host: nothing here reaches a GPU."""
import ctypes as C
import math

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import build
    if build.is_stale():
        build.build()
    from paper_2602_01665_amd import binding
    return binding


FAKE = 0x100000          # an address that is only looked at
NULL, SHAPE, ALIGN, PARAM = -1, -2, -3, -5


def rows(B, stride, type=0, data=FAKE):
    return C.byref(B.TabxRows(data, stride, type))


def heads(B, tick=1 << 20, row=1 << 10, head=1 << 5, type=0, data=FAKE):
    return C.byref(B.TabxHeads(data, tick, row, head, type))


def test_rms_norm(B):
    def call(n=4, width=8, x=rows(B, 8), res=None, weight=FAKE, eps=1e-5, total=None, y=rows(B, 8), scale=None, rstd=FAKE):
        return B._lib.tabx_rms_norm(n, width, x, res, None, weight, eps, total, y, scale, rstd, None)

    assert call(n=0, x=None, y=None, rstd=None) == 0
    for kw in (dict(n=-1), dict(n=(1 << 40) + 1), dict(width=0), dict(width=8193), dict(x=rows(B, 7)), dict(y=rows(B, 7)), dict(res=rows(B, 7)),
               dict(total=rows(B, 7)), dict(x=rows(B, 8, 3)), dict(res=rows(B, 8, 3)), dict(total=rows(B, 8, 3)), dict(y=rows(B, 8, 4)),
               dict(x=rows(B, 8, 4)), dict(scale=FAKE), dict(n=1 << 30, x=rows(B, 1 << 33))):
        assert call(**kw) == SHAPE, kw
    for eps in (-1e-9, math.nan, math.inf):
        assert call(eps=eps) == PARAM
    for kw in (dict(x=None), dict(y=None), dict(y=rows(B, 8, 3)), dict(x=rows(B, 8, 0, None)), dict(y=rows(B, 8, 3, None), scale=FAKE)):
        assert call(**kw) == NULL, kw
    for kw in (dict(x=rows(B, 8, 0, FAKE + 2)), dict(res=rows(B, 8, 1, FAKE + 1)), dict(total=rows(B, 8, 2, FAKE + 1)), dict(weight=FAKE + 2),
               dict(rstd=FAKE + 1), dict(y=rows(B, 8, 3, FAKE + 1), scale=FAKE + 2)):
        assert call(**kw) == ALIGN, kw


def test_rms_norm_backward(B):
    def call(n=64, width=8, s=rows(B, 8), gy=rows(B, 8), gs=None, gx=rows(B, 8), gw=FAKE, ws=FAKE, size=1 << 20, rstd=FAKE, weight=None):
        return B._lib.tabx_rms_norm_backward(n, width, s, None, weight, rstd, gy, gs, gx, gw, ws, size, None)

    need = B.tabx_rms_norm_workspace
    assert need(0, 8) > 0 and need(1 << 30, 368) == need(1 << 24, 368) <= 1024 * 368 * 4
    assert call(n=0, s=None, gy=None, gx=None, gw=None, ws=None, rstd=None) == 0
    for kw in (dict(n=-1), dict(width=0), dict(width=8193), dict(size=need(64, 8) - 1), dict(gx=rows(B, 7)), dict(gy=rows(B, 8, 9)),
               dict(gs=rows(B, 8, 1)), dict(gs=rows(B, 7)), dict(s=rows(B, 8, 3))):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(ws=None), dict(gw=None, gx=None), dict(rstd=None), dict(gy=None), dict(s=None)):
        assert call(**kw) == NULL, kw
    for kw in (dict(ws=FAKE + 8), dict(gw=FAKE + 2), dict(rstd=FAKE + 1), dict(weight=FAKE + 3), dict(gx=rows(B, 8, 1, FAKE + 1))):
        assert call(**kw) == ALIGN, kw
    for n, width in ((-1, 8), (4, 0), (4, 8193), (2 ** 64 + 4, 8), (4, 2 ** 32 + 8)):
        with pytest.raises(B.TabxError):
            need(n, width)


def test_rotary(B):
    def axes(*of):
        return (B.TabxAxis * len(of))(*[B.TabxAxis(*a) for a in of])

    def call(n=6, h=2, width=16, x=None, y=None, a=None, count=None, freq=FAKE):
        x, y = x or heads(B, 0, 64, 16), y or heads(B, 0, 64, 16)
        a = axes((FAKE, 4, 1, 4), (FAKE, 0, 3, 4)) if a is None else a
        return B._lib.tabx_rotary(n, h, width, x, None, a, len(a) if count is None else count, freq, 0, 0, y, None)

    assert call(n=0, a=axes((None, 4, 1, 4)), freq=None) == 0
    for kw in (dict(n=-1), dict(h=0), dict(width=1), dict(width=513), dict(count=0), dict(count=5), dict(a=axes((FAKE, 4, 1, 9))),
               dict(a=axes((FAKE, 4, 1, 4), (FAKE, 0, 1, 5))), dict(a=axes((FAKE, 4, 1, 0))), dict(a=axes((FAKE, 4, 1, -1))),
               dict(a=axes((FAKE, 1, 1, 4))), dict(a=axes((FAKE, 4, 0, 4))), dict(a=axes((FAKE, 4, 4, 4))),
               dict(a=axes((FAKE, 4, 1, 2 ** 31 - 1), (FAKE, 4, 1, 2 ** 31 - 1))),
               dict(x=heads(B, 0, 64, 16, 3)), dict(x=heads(B, 0, 64, 16, 1)), dict(x=heads(B, 0, -64, 16)), dict(x=heads(B, 0, 1 << 60, 16)),
               dict(y=heads(B, 0, 31, 16)), dict(y=heads(B, 0, 64, 15)), dict(y=heads(B, 0, 0, 16)), dict(y=heads(B, 0, 16, 16)),
               dict(h=1 << 27, width=16), dict(x=heads(B, 0, 96, 16)), dict(x=heads(B, 0, 64, 24))):
        assert call(**kw) == SHAPE, kw
    assert call(x=heads(B, 0, 64, 16, 0, None)) == NULL and call(freq=None) == NULL and call(a=axes((None, 4, 1, 4))) == NULL
    assert B._lib.tabx_rotary(6, 2, 16, None, None, axes((FAKE, 4, 1, 4)), 1, FAKE, 0, 0, heads(B, 0, 64, 16), None) == NULL
    assert B._lib.tabx_rotary(6, 2, 16, heads(B), None, None, 1, FAKE, 0, 0, heads(B, 0, 64, 16), None) == NULL
    assert call(freq=FAKE + 4) == ALIGN and call(a=axes((FAKE + 2, 4, 1, 4))) == ALIGN and call(y=heads(B, 0, 64, 16, 0, FAKE + 2)) == ALIGN


def test_linear_attention(B):
    lib = B._lib
    h = lambda **kw: heads(B, **kw)  # noqa: E731

    def step(n=6, H=2, K=16, V=16, q=h(), k=h(), v=h(), decay=FAKE, scale=1.0, units=1, state=FAKE, out=h()):
        return lib.tabx_linear_attention_step(n, H, K, V, q, k, v, decay, scale, None, units, None, state, out, None)

    def many(T=5, n=6, H=2, K=16, V=16, q=h(), k=h(), v=h(), decay=FAKE, scale=1.0, units=1, s=FAKE, t=FAKE, out=h(), ws=None, size=0):
        return lib.tabx_linear_attention(T, n, H, K, V, q, k, v, decay, scale, None, units, None, s, t, out, ws, size, None)

    def back(T=5, n=6, H=2, K=16, V=16, q=h(), k=h(), v=h(), decay=FAKE, scale=1.0, units=1, s=FAKE, gs=FAKE, go=h(), gq=h(), gk=h(), gv=h(),
             gi=FAKE, ws=None, size=0):
        return lib.tabx_linear_attention_backward(T, n, H, K, V, q, k, v, decay, scale, None, units, None, s, gs, go, gq, gk, gv, gi, ws, size, None)

    assert step(n=0, q=None, k=None, v=None, decay=None, state=None, out=None) == 0
    assert many(n=0, q=None, k=None, v=None, decay=None, out=None) == 0 and many(T=0, q=None, out=None, t=None) == 0
    assert back(n=0, q=None, decay=None, go=None) == 0 and back(T=0, q=None, go=None, gi=None) == 0
    for call in (step, many, back):
        for kw in (dict(n=-1), dict(H=0), dict(H=65537), dict(n=1 << 31), dict(n=1 << 16, H=1 << 15), dict(K=0), dict(K=129), dict(V=0), dict(V=129),
                   dict(units=0), dict(units=4), dict(q=h(type=3)), dict(k=h(type=1)), dict(v=h(type=2)), dict(q=h(row=-8)),
                   dict(k=h(row=1 << 60))):
            assert call(**kw) == SHAPE, (call, kw)
        for scale in (math.nan, math.inf, -math.inf):
            assert call(scale=scale) == PARAM
        for kw in (dict(q=None), dict(k=None), dict(v=h(data=None)), dict(decay=None)):
            assert call(**kw) == NULL, (call, kw)
        for kw in (dict(q=h(data=FAKE + 2)), dict(decay=FAKE + 1)):
            assert call(**kw) == ALIGN, (call, kw)
    # outputs whose elements share a place
    for o in (h(head=15), h(row=16), h(head=0), h(row=32, head=32)):
        assert step(out=o) == SHAPE and many(out=o) == SHAPE
    for o in (h(tick=1 << 10), h(tick=0), h(tick=1 << 60)):
        assert many(out=o) == SHAPE and back(gq=o) == SHAPE and back(gk=o) == SHAPE and back(gv=o) == SHAPE
    assert many(T=-1) == SHAPE and many(T=(1 << 30) + 1) == SHAPE and back(gk=h(type=1)) == SHAPE
    assert step(state=None) == NULL and step(out=None) == NULL and many(out=None) == NULL and back(go=None) == NULL
    assert back(gq=None, gk=None, gv=None, gi=None) == NULL
    assert step(state=FAKE + 2) == ALIGN and many(s=FAKE + 1) == ALIGN and many(t=FAKE + 2) == ALIGN and back(gs=FAKE + 1) == ALIGN and back(gi=FAKE + 3) == ALIGN
    # few rows of many ticks need room
    need = B.tabx_linear_attention_workspace(100000, 2, 2, 16, 16)
    assert need > 0 and B.tabx_linear_attention_workspace(100000, 1 << 16, 2, 16, 16) == 0 == B.tabx_linear_attention_workspace(8, 1, 1, 16, 16)
    assert B.tabx_linear_attention_workspace(0, 0, 1, 1, 1) == 0
    for call in (many, back):
        big = dict(T=100000, n=2, **{n: h(tick=1 << 12) for n in ("q", "k", "v")})
        assert call(ws=None, **big) == NULL and call(ws=FAKE + 8, size=need, **big) == ALIGN and call(ws=FAKE, size=need - 1, **big) == SHAPE
    for bad in ((-1, 2, 2, 4, 4), (4, -1, 2, 4, 4), ((1 << 30) + 1, 2, 2, 4, 4), (4, 2, 0, 4, 4), (4, 2, 2 ** 32 + 2, 4, 4), (4, 2, 2, 2 ** 32 + 4, 4),
                (2 ** 64, 2, 2, 4, 4)):
        with pytest.raises(B.TabxError):
            B.tabx_linear_attention_workspace(*bad)


def test_tensors_are_checked_before_their_addresses_are_taken(B):
    f, u8 = torch.float32, torch.uint8

    def refused(why, call, *args, **kw):
        with pytest.raises(B.TabxError, match=why):
            call(*args, **kw)

    x, y, w = torch.zeros(6, 16), torch.zeros(6, 16), torch.ones(16)
    norm, q8 = B.tabx_rms_norm, torch.zeros(6, 16).to(torch.float8_e4m3fn)
    refused("not on a GPU", norm, x, w, 1e-5, y)
    refused("not on a GPU", norm, x, w, 1e-5, q8, torch.zeros(6))
    refused("8 bits", norm, x, w, 1e-5, q8)
    refused("8 bits", norm, x, w, 1e-5, y, torch.zeros(6))
    refused("float8", norm, q8, w, 1e-5, y)
    refused("not one of", norm, x.double(), w, 1e-5, y)
    refused("residual has 5 rows", norm, x, w, 1e-5, y, residual=y[:5])
    refused("sum has rows of 15", norm, x, w, 1e-5, y, residual=y, sum=y[:, :15])
    refused("rstd has 5", norm, x, w, 1e-5, y, None, torch.zeros(5))
    refused("row_mask", norm, x, w, 1e-5, y, row_mask=torch.zeros(6, dtype=torch.bool))
    back, r, ws = B.tabx_rms_norm_backward, torch.zeros(6), torch.zeros(1 << 12, dtype=u8)
    refused("not on a GPU", back, x, w, r, y, None, y, w, ws)
    refused("rstd is needed", back, x, w, None, y, None, y)
    refused("grad_sum has 5", back, x, w, r, y, y[:5], y)
    refused("float64", back, x, w, r, y, None, y, w.double(), ws)

    h, freq, t = torch.zeros(6, 2, 8), torch.ones(4, dtype=torch.float64), torch.zeros(6, dtype=torch.int32)
    rot = B.tabx_rotary
    refused("not on a GPU", rot, h, [(t, 4)], freq, h)
    refused("not on a GPU", rot, h, [(t[:2], 4)], freq, h)
    refused("does not divide", rot, h, [(t[:4], 4)], freq, h)
    refused("does not divide", rot, h, [(t[:0], 4)], freq, h)
    refused("int64", rot, h, [(t.long(), 4)], freq, h)
    refused("frequency has 4", rot, h, [(t, 3)], freq, h)
    refused("frequency is torch.float32", rot, h, [(t, 4)], freq.float(), h)
    refused("0 axes", rot, h, [], freq, h)
    refused("5 axes", rot, h, [(t, 1)] * 5, freq, h)
    refused("y has 6 rows of 2 heads of 7", rot, h, [(t, 4)], freq, h[..., :7])
    refused("equal distances", rot, torch.zeros(3, 4, 2, 8)[:, :2], [(t, 4)], freq, h)
    refused("next to each other", rot, torch.zeros(6, 8, 2).transpose(1, 2), [(t, 4)], freq, h)
    refused("pairs", rot, h, [(t, -1)], freq, h)

    T, R, H, K, V = 5, 6, 2, 8, 4
    q, k, v = torch.zeros(T, R, H, K), torch.zeros(T, R, H, K), torch.zeros(T, R, H, V)
    decay, s, fresh = torch.zeros(H), torch.zeros(R, H, K, V), torch.zeros(T, 2, dtype=u8)
    many, step, grad = B.tabx_linear_attention, B.tabx_linear_attention_step, B.tabx_linear_attention_backward
    refused("not on a GPU", many, q, k, v, decay, 1.0, v, fresh, s, s)
    refused("k has 5 ticks|k has 4 ticks", many, q, k[:4], v, decay, 1.0, v)
    refused("k has 6 rows of 2 heads of 7", many, q, k[..., :7], v, decay, 1.0, v)
    refused("out has 5 rows", many, q, k, v, decay, 1.0, v[:, :5])
    refused("log_decay has 3", many, q, k, v, torch.zeros(3), 1.0, v)
    refused("log_decay is needed", many, q, k, v, None, 1.0, v)
    refused("do not share", many, q, k, v, decay, 1.0, v, torch.zeros(T, 4, dtype=u8))
    refused("do not share", many, q, k, v, decay, 1.0, v, torch.zeros(3, dtype=u8))
    refused("fresh is torch.bool", many, q, k, v, decay, 1.0, v, fresh.bool())
    refused("state_in has", many, q, k, v, decay, 1.0, v, fresh, s[:5])
    refused("state_out is torch.bfloat16", many, q, k, v, decay, 1.0, v, fresh, s, s.bfloat16())
    refused("controlled has 5", many, q, k, v, decay, 1.0, v, controlled=torch.zeros(5, dtype=u8))
    refused("dimensions", many, q[0, 0], k, v, decay, 1.0, v)
    refused("not on a GPU", step, q[0], k[0], v[0], decay, 1.0, s, v[0], fresh[0])
    refused("state is needed", step, q[0], k[0], v[0], decay, 1.0, None, v[0])
    refused("state is not contiguous", step, q[0], k[0], v[0], decay, 1.0, s.transpose(2, 3).contiguous().transpose(2, 3), v[0])
    refused("not on a GPU", grad, q, k, v, decay, 1.0, v, q, k, v, fresh, s, s, s)
    refused("grad_v has 6 rows of 2 heads of 8", grad, q, k, v, decay, 1.0, v, q, k, q)
    refused("grad_state_in has", grad, q, k, v, decay, 1.0, v, q, k, v, None, s, s, s[1:])


def test_a_batch_refuses_turns_of_other_axes(B):
    from paper_2602_01665_amd import inputs as I
    w = I.WORKLOADS["c2_4096env_5v5"]
    env = B.TabxEnv(I.make_params(w, 4), I.make_scenario(w, 4), device="cpu")
    x = torch.zeros(4, env.N, 2, 12)
    freq = torch.ones(6, dtype=torch.float64)
    for batch in [env] + env.parts(1):
        with pytest.raises(B.TabxError, match="2 axes"):
            batch.rotate(x, (3, 3), freq, x)
        with pytest.raises(B.TabxError, match="not on a GPU"):
            batch.rotate(x, (2, 2, 2), freq, x)
        q, s = torch.zeros(4, env.N, 2, 8), torch.zeros(4, env.N, 2, 8, 8)
        with pytest.raises(B.TabxError, match="not on a GPU"):
            batch.remember(q, q, q, torch.zeros(2), 1.0, s, q)
        with pytest.raises(B.TabxError, match="state has"):
            batch.remember(q, q, q, torch.zeros(2), 1.0, s[:3], q)


def test_a_batch_refuses_heads_of_other_rows(B):
    """Ticks, places and ended episodes would be dealt out to them as if they were fewer, larger envs."""
    from paper_2602_01665_amd import inputs as I
    w = I.WORKLOADS["c2_4096env_5v5"]
    env = B.TabxEnv(I.make_params(w, 4), I.make_scenario(w, 4), device="cpu")
    freq, decay = torch.ones(6, dtype=torch.float64), torch.zeros(2)
    for batch in [env] + env.parts(2):
        E, N = batch.E, env.N
        for lead in ((2 * E, N), (E, 2 * N), (3 * E * N,), (E, N, 2), (1, E * N + E)):
            x, s = torch.zeros(*lead, 2, 12), torch.zeros(*lead, 2, 12, 12)
            with pytest.raises(B.TabxError, match=f"rotate.*rows of heads, not {E} x {N}"):
                batch.rotate(x, (2, 2, 2), freq, x)
            with pytest.raises(B.TabxError, match=f"remember.*rows of heads, not {E} x {N}"):
                batch.remember(x, x, x, decay, 1.0, s, x)
        for lead in ((E, N), (E * N,)):
            x, s = torch.zeros(*lead, 2, 12), torch.zeros(*lead, 2, 12, 12)
            with pytest.raises(B.TabxError, match="not on a GPU"):
                batch.rotate(x, (2, 2, 2), freq, x)
            with pytest.raises(B.TabxError, match="not on a GPU"):
                batch.remember(x, x, x, decay, 1.0, s, x)
        with pytest.raises(B.TabxError, match="rows of heads"):
            batch.rotate(torch.zeros(12), (2, 2, 2), freq, torch.zeros(12))
