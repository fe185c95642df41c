"""The calls of a unit's memory in 64 bits, from their definitions, and how far 32 bits may be off.

U is half a step of float32, relative.  A sum of n terms in any order is off by at most (n - 1) U times
the sum of the terms' magnitudes."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
# half a step, relative; and half the smallest step there is
STEP = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134),
        torch.float16: (2.0 ** -11, 2.0 ** -25), torch.float8_e4m3fn: (2.0 ** -4, 2.0 ** -10)}
# additions one value passes through in a norm's sum: its lane's pieces (at most four of four
# elements), six steps across a wavefront, sixteen wavefronts
CHAIN = 4 * 4 + 6 + 16


def f64(t):
    return t.detach().cpu().double()


def rounded(bound, value, dtype):
    """bound on a 32-bit result turned into one on its rounding to dtype."""
    rel, least = STEP[dtype]
    return bound + rel * (value.abs() + bound) + least


def near(got, want, bound, what):
    got = f64(got)
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), what
    off, bound = (got - want).abs()[fine], bound.expand(want.shape)[fine]
    over = off > bound
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} off, by up to {float((off / bound.clamp(min=1e-300)).max()):.3g} bounds"


# --- root-mean-square norm ---------------------------------------------------------------------------

def norm(x, residual, weight, eps, sum_type, out_type):
    """{name: (value, bound)} of rows [R, W] of 32 bits or fewer."""
    W = x.shape[1]
    s = f64(x)
    d_s = torch.zeros_like(s)
    if residual is not None:
        s = s + f64(residual)
        d_s = U * s.abs()
    out = {}
    if sum_type is not None:
        out["sum"] = (s, rounded(d_s, s, sum_type))
        # the rounding of the sum is part of the definition: 32 bits of it, then its type
        s = s.float().to(sum_type).double()
        d_s = torch.zeros_like(s)
    w = torch.ones(W, dtype=torch.float64) if weight is None else f64(weight)
    mean = (s * s).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(mean + eps)
    d_mean = (CHAIN + 4) * U * mean + 2 * (d_s * s.abs()).mean(1, keepdim=True)
    rel = 0.5 * d_mean / (mean + eps) + 6 * U
    out["rstd"] = (rstd[:, 0], (rstd * rel)[:, 0])
    y = s * rstd * w
    d_y = y.abs() * (rel + 4 * U) + d_s * (rstd * w).abs()
    if out_type is torch.float8_e4m3fn:
        most = y.abs().amax(1, keepdim=True)
        scale = torch.clamp(most / 448.0, min=2.0 ** -126)
        d_scale = d_y.amax(1, keepdim=True) / 448.0 + 2 * U * scale
        out["scale"] = (scale[:, 0], d_scale[:, 0])
        d_y = (d_y + y.abs() * (d_scale / scale + 4 * U)) / scale
        y = y / scale
    out["y"] = (y, rounded(d_y, y, out_type))
    return out


def norm_grad(s, weight, rstd, gy, gs, on, out_type, turns):
    """{name: (value, bound)}; turns: rows that one lane adds up, behind which come at most 64 additions."""
    W = s.shape[1]
    s, rstd, gy = f64(s), f64(rstd)[:, None], f64(gy)
    w = torch.ones(W, dtype=torch.float64) if weight is None else f64(weight)
    h = s * rstd
    g = gy * w
    b = (g * h).mean(1, keepdim=True)
    gx = rstd * (g - h * b)
    d_b = (CHAIN + 8) * U * (g * h).abs().mean(1, keepdim=True)
    d = rstd * (h.abs() * d_b + 6 * U * (g.abs() + (h * b).abs()))
    if gs is not None:
        gx = gx + f64(gs)
        d = d + U * gx.abs()
    keep = on[:, None]
    zero = torch.zeros((), dtype=torch.float64)
    d = torch.where(keep, rounded(d, gx, out_type), zero)
    hk, gk = torch.where(keep, h, zero), torch.where(keep, gy, zero)
    return {"grad_x": (torch.where(keep, gx, zero), d),
            "grad_weight": ((hk * gk).sum(0), (turns + 64 + 4) * U * (hk * gk).abs().sum(0) + 2.0 ** -140)}


# --- rotation ----------------------------------------------------------------------------------------

def rotary(x, axes, frequency, interleaved, inverse):
    """(value, bound) of x [R, H, W]; axes: (positions, pairs)."""
    R = x.shape[0]
    v, at, parts, far = f64(x), 0, [], []
    for position, pairs in axes:
        p = f64(position).flatten()
        p = p.repeat_interleave(R // p.numel())
        parts.append(p[:, None] * f64(frequency)[at:at + pairs])
        at += pairs
    a = torch.cat(parts, 1) * (-1.0 if inverse else 1.0)
    P = a.shape[1]
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    i = torch.arange(P)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + P)
    out, bound = v.clone(), torch.zeros_like(v)
    m, n = v[..., first], v[..., second]
    out[..., first], out[..., second] = m * c - n * s, m * s + n * c
    # cosine and sine: five steps of 32 bits at most, and the angle's own three roundings in 64
    d = 5 * U + 3 * 2.0 ** -53 * a.abs()[:, None]
    both = (d + 3 * U) * (m.abs() + n.abs())
    bound[..., first], bound[..., second] = both, both
    return out, rounded(bound, out, x.dtype)


# --- linear attention --------------------------------------------------------------------------------

SPLIT = 2.0 ** -16             # what 16-bit operands in two parts leave of a 32-bit one


def _gamma(log_decay):
    g = f64(log_decay)
    return torch.exp(torch.where(g < 0.0, g, torch.zeros_like(g)))[:, None, None]


def _fresh(fresh, T, R):
    if fresh is None:
        return torch.zeros(T, R, dtype=torch.bool)
    f = fresh.cpu().reshape(T, -1) != 0
    return f.repeat_interleave(R // f.shape[1], 1)


def _walk(x, y, state, gamma, fresh, order):
    """For every tick in order: the state behind it, which forgets, fades and takes x y^T in."""
    T, R, H, K = x.shape
    S = torch.zeros(R, H, K, y.shape[-1], dtype=torch.float64) if state is None else state.clone()
    for t in order:
        S = torch.where(fresh[t][:, None, None, None], torch.zeros((), dtype=torch.float64), S * gamma)
        S = S + x[t][..., :, None] * y[t][..., None, :]
        yield t, S
    yield None, S


def _loose(T, K, log_decay, dtype):
    """Roundings of a term, relative: an addition for every tick, the dot product, powers of the decay (whose
    exponent is rounded, and which are nothing where it is above 104), and split operands where they are."""
    g = f64(log_decay)
    g = torch.where(torch.isfinite(g), g, torch.full_like(g, -104.0)).clamp(max=0.0)
    powers = 4.0 * (-g * T).clamp(max=104.0)
    return (((K + T + 40) + powers) * U + (0.0 if dtype is torch.float32 else 4 * SPLIT))[:, None]


def attention(q, k, v, log_decay, scale, fresh, state):
    """{name: (value, bound)} of q, k [T, R, H, K] and v [T, R, H, V]."""
    T, R, H, K = q.shape
    V = v.shape[-1]
    x, y, z, begins, gamma = f64(q), f64(k), f64(v), _fresh(fresh, T, R), _gamma(log_decay)
    s0 = None if state is None else f64(state)
    out, mag = torch.zeros(T, R, H, V, dtype=torch.float64), torch.zeros(T, R, H, V, dtype=torch.float64)
    for t, S in _walk(y, z, s0, gamma, begins, range(T)):
        if t is not None:
            out[t] = scale * (x[t][..., :, None] * S).sum(-2)
    final = S
    for t, S in _walk(y.abs(), z.abs(), None if s0 is None else s0.abs(), gamma, begins, range(T)):
        if t is not None:
            mag[t] = abs(scale) * (x[t].abs()[..., :, None] * S).sum(-2)
    loose = _loose(T, K, log_decay, q.dtype)
    tiny = 2.0 ** -120
    exact = _loose(T, K, log_decay, torch.float32)             # the state is kept in 32 bits, whatever goes in
    return {"out": (out, rounded(loose * mag + tiny, out, q.dtype)),
            "state_out": (final, exact[..., None] * S + tiny)}


def attention_grad(q, k, v, log_decay, scale, fresh, state, grad_out, grad_state):
    """{name: (value, bound)} from the recurrences of S and D."""
    T, R, H, K = q.shape
    begins, gamma = _fresh(fresh, T, R), _gamma(log_decay)
    loose = _loose(T, max(K, v.shape[-1]), log_decay, q.dtype)
    tiny = 2.0 ** -120

    def run(of):
        x, y, z, g = (of(f64(a)) for a in (q, k, v, grad_out))
        c = scale if of is _same else abs(scale)
        s0 = None if state is None else of(f64(state))
        gq, gk, gv = torch.zeros_like(x), torch.zeros_like(y), torch.zeros_like(z)
        for t, S in _walk(y, z, s0, gamma, begins, range(T)):
            if t is not None:
                gq[t] = c * (S * g[t][..., None, :]).sum(-1)
        D = torch.zeros(R, H, K, v.shape[-1], dtype=torch.float64) if grad_state is None else of(f64(grad_state))
        for t in range(T - 1, -1, -1):
            D = D + c * x[t][..., :, None] * g[t][..., None, :]
            gk[t], gv[t] = (D * z[t][..., None, :]).sum(-1), (D * y[t][..., :, None]).sum(-2)
            D = torch.where(begins[t][:, None, None, None], torch.zeros((), dtype=torch.float64), D * gamma)
        return {"grad_q": gq, "grad_k": gk, "grad_v": gv, "grad_state_in": D}

    value, mag = run(_same), run(torch.abs)
    out = {n: (value[n], rounded(loose * mag[n] + tiny, value[n], q.dtype)) for n in ("grad_q", "grad_k", "grad_v")}
    exact = _loose(T, max(K, v.shape[-1]), log_decay, torch.float32)
    out["grad_state_in"] = (value["grad_state_in"], exact[..., None] * mag["grad_state_in"] + tiny)
    return out


def _same(x):
    return x


def decays(H):
    return torch.log1p(-(2.0 ** -(1.0 + torch.arange(H) * (6.0 / H)))).float()


assert math.isclose(float(torch.exp(decays(1))[0]), 0.5)
