"""The learner's calls in 64 bits, one row at a time in plain numpy, and how far 32 bits may be off.

U is half a step of float32.  A sum of n terms in any order is off by at most (n - 1) U times the
sum of the terms' magnitudes; where it is taken over lanes and pieces, n is the length of the
longest chain of additions.
"""
from __future__ import annotations

import numpy as np
import torch

U = 2.0 ** -24
ATTACK, CHOICES = 5, 8
# half a step, relative; and half the smallest step there is
STEP = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134),
        torch.float16: (2.0 ** -11, 2.0 ** -25)}
# additions one value passes through in a row's sum: its lane's pieces (at most four of four
# elements), six steps across a wavefront, sixteen wavefronts
CHAIN = 4 * 4 + 6 + 16


def f64(t):
    return t.detach().to("cpu").double().numpy()


def rounded(bound, value, dtype):
    """bound on a 32-bit result turned into one on its rounding to dtype."""
    rel, least = STEP[dtype]
    return bound + rel * (np.abs(value) + bound) + least


def norm(x, weight, bias, eps, dtype):
    """(y, mean, rstd, bounds of the three) of rows x [R, W] in float64."""
    W = x.shape[1]
    w = np.ones(W) if weight is None else weight
    b = np.zeros(W) if bias is None else bias
    mean = x.mean(1, keepdims=True)
    c = x - mean
    var = (c * c).mean(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd = 1.0 / np.sqrt(var + eps)
    y = c * rstd * w + b
    d_mean = (CHAIN + 2) * U * np.abs(x).mean(1, keepdims=True)
    # c is off by d_mean and its own rounding; in the variance the first counts squared, as the c
    # sum to zero, the sum's chain and three roundings relatively
    d_c = d_mean + U * np.abs(c)
    d_var = d_mean ** 2 + 2 * d_mean * U * np.abs(c).mean(1, keepdims=True) + (CHAIN + 8) * U * var
    rel = 0.5 * d_var / (var + eps) + 6 * U
    d_rstd = rstd * rel
    d_y = np.abs(w) * (rstd * d_c * (1 + rel) + np.abs(c) * d_rstd) + 4 * U * (np.abs(c * rstd * w) + np.abs(b))
    return y, mean[:, 0], rstd[:, 0], rounded(d_y, y, dtype), d_mean[:, 0], d_rstd[:, 0]


def norm_grad(x, on, weight, mean, rstd, gy, dtype, turns):
    """(grad_x, grad_weight, grad_bias, bounds of the three); `mean` and `rstd` are inputs.  turns:
    rows that one lane adds up, behind which come at most 64 joining additions."""
    W = x.shape[1]
    w = np.ones(W) if weight is None else weight
    h = (x - mean[:, None]) * rstd[:, None]
    g = gy * w
    a, b = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    gx = rstd[:, None] * (g - a - h * b)
    mag_a, mag_b = np.abs(g).mean(1, keepdims=True), np.abs(g * h).mean(1, keepdims=True)
    d_a, d_b = (CHAIN + 4) * U * mag_a, (CHAIN + 8) * U * mag_b
    d_gx = rstd[:, None] * (d_a + np.abs(h) * d_b + 8 * U * (np.abs(g) + np.abs(a) + np.abs(h * b)))
    keep = on[:, None]
    gx, d_gx = np.where(keep, gx, 0.0), np.where(keep, rounded(d_gx, gx, dtype), 0.0)
    gyk, hk = np.where(keep, gy, 0.0), np.where(keep, h, 0.0)
    chain = (turns + 64 + 4) * U
    return (gx, (gyk * hk).sum(0), gyk.sum(0), d_gx,
            chain * np.abs(gyk * hk).sum(0) + 2.0 ** -140, chain * np.abs(gyk).sum(0) + 2.0 ** -140)


def allowed(logits, action_mask=None):
    """Scores with -infinity for what cannot be chosen (NaN included)."""
    l = np.array(logits, dtype=np.float64)
    if action_mask is not None:
        l[action_mask == 0, ATTACK] = -np.inf
    l[np.isnan(l)] = -np.inf
    return l


def weights(l, temperature):
    """exp((l - max) / temperature) of one row, and (l - max) / temperature."""
    top = l.max()
    if top == -np.inf:
        return None, None
    with np.errstate(invalid="ignore"):
        d = np.where(l == top, 0.0, (l - top) / temperature)
    return np.exp(d), d


def choose(l, temperature, top_k, top_p, min_p, u):
    """Index drawn from one row of scores, None if there is nothing to choose."""
    top = l.max()
    if top == -np.inf:
        return None
    if temperature == 0.0:
        return int(np.argmax(l))                       # the first of the largest
    w, _ = weights(l, temperature)
    order = np.argsort(-l, kind="stable")
    order = order[np.isfinite(-l[order]) | (l[order] == np.inf)]
    if top_k:
        order = order[:top_k]
    if top_p < 1.0:
        upto = np.cumsum(w[order])
        order = order[(upto - w[order]) < np.float64(np.float32(top_p)) * upto[-1]]
    order = order[w[order] >= np.float64(np.float32(min_p))]
    kept = np.zeros_like(w)
    kept[order] = w[order]
    upto = np.cumsum(kept)
    u = np.float32(u)
    u = np.float32(0.0) if not u > 0 else min(u, np.float32(1 - 2.0 ** -24))
    return int(np.argmax(upto > np.float64(u) * upto[-1]))


def shares(l, temperature):
    """(d, p, log p, entropy, bound of log p_i and of p_i relatively) of rows of scores; a row with
    nothing to choose has p = 0."""
    top = l.max(1, keepdims=True)
    some = top > -np.inf
    with np.errstate(invalid="ignore"):
        d = np.where(l == top, 0.0, (l - top) / temperature)
    d = np.where(some, d, -np.inf)
    e = np.exp(d)
    total = np.where(some, e.sum(1, keepdims=True), 1.0)
    p = e / total
    logp = d - np.log(total)
    logp[logp < -np.finfo(np.float32).max] = -np.inf    # beyond what 32 bits hold
    info = np.where(p > 0, -p * np.where(p > 0, logp, 0.0), 0.0)
    fin = np.where(np.isfinite(d), d, 0.0)
    # a weight is off by three roundings of its exponent and two steps of exp
    delta = 4 * U * np.abs(fin) + 4 * U * (p * np.abs(fin)).sum(1, keepdims=True) + 16 * U
    return fin, p, logp, info.sum(1), delta, some[:, 0]


def log_prob(l, actions, temperature):
    """(log_prob, entropy, their bounds) of rows of scores."""
    a = np.where(actions < CHOICES, actions, 0).astype(np.int64)
    _, p, logp, h, delta, some = shares(l, temperature)
    at = np.arange(len(a))
    lp = np.where(some, logp[at, a], 0.0)
    mag = np.where(np.isfinite(logp), np.abs(logp), 0.0)
    d_lp = delta[at, a] + 4 * U * mag[at, a]
    d_h = (p * (delta * mag + delta) + 16 * U * p * mag).sum(1) + 2.0 ** -120
    return lp, np.where(some, h, 0.0), d_lp, d_h


def log_prob_grad(l, actions, temperature, gl, ge, dtype):
    """(grad_logits, its bound)."""
    a = np.where(actions < CHOICES, actions, 0).astype(np.int64)
    _, p, logp, h, delta, some = shares(l, temperature)
    _, _, _, d_h = log_prob(l, actions, temperature)
    at = np.arange(len(a))
    taken = logp[at, a]
    gl = np.where(np.isfinite(taken) & some, gl, 0.0)[:, None]
    one = np.zeros_like(p)
    one[at, a] = 1.0
    fin = np.where(p > 0, np.where(np.isfinite(logp), logp, 0.0), 0.0)
    # 1 - p_a as the sum of the others: taken from 1 in 64 bits, what is left of 1e-20 would be 1e-16
    rest = ((1 - one) * p).sum(1, keepdims=True)
    toward = np.where(one > 0, rest, -p)
    even = p * (fin + h[:, None])
    g = (gl * toward - ge[:, None] * even) / temperature
    d_toward = np.where(one > 0, ((1 - one) * p * (delta + 8 * U)).sum(1, keepdims=True), p * (delta + 4 * U))
    d_even = p * delta * np.abs(fin + h[:, None]) + p * (delta + 4 * U * np.abs(fin) + d_h[:, None]) + 4 * U * np.abs(even)
    # (a share below 2^-126 may be lost)
    bound = (np.abs(gl) * (d_toward + 2.0 ** -120) + np.abs(ge[:, None]) * (d_even + 2.0 ** -110)) / temperature
    bound = bound + 6 * U * (np.abs(gl * toward) + np.abs(ge[:, None] * even)) / temperature + 2.0 ** -120
    g = np.where(some[:, None], g, 0.0)
    return g, np.where(some[:, None], rounded(bound, g, dtype), 0.0)


def near(got, want, bound, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    off = np.abs(got[fine] - want[fine])
    over = off > bound[fine]
    assert not over.any(), f"{what}: {int(over.sum())} of {over.size} off, by up to {float((off / np.maximum(bound[fine], 1e-300)).max()):.3g} bounds"
