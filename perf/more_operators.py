"""The calls of a unit's memory whose speed counts, with inputs as a training program has them: a
residual stream's root-mean-square norm and its gradients, rotation of queries and keys by tick and
place, linear attention with a decay for each head over a unit's ticks (one tick of a rollout, many
ticks of an update) and its gradients.

`run` makes the library's calls where `own` is true and computes the same from elementary tensor
operations where it is false.  `exact` evaluates the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-5
LARGEST = 448.0                # of the 8-bit type
SMALLEST_SCALE = 2.0 ** -126
# rows = envs x units (the norm's and the rotation's: x ticks); `controlled`: only the first half of
# each env's units learns; `joined`: queries, keys and values are columns of one projection's output
BASE = dict(op="", rows=0, units=1, ticks=1, width=0, heads=1, key=0, value=0, type="f32", out="f32",
            pad=0, controlled=False, residual=True, stream=False, axes=3, pairs=0, interleaved=False,
            inverse=False, first_tick=0, joined=True, ends=0.0, state=True)


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # a handful of duels played by a network: launch and latency bound
        _case("norm 3v3 x16", op="norm", rows=16 * 6, units=6, width=128, type="bf16", out="bf16"),
        # the headline batch, half of whose units learn, to 8 bits for the next product
        _case("norm 10v10 x16384 to 8 bits", op="norm", rows=16384 * 20, units=20, width=512,
              type="bf16", out="e4m3", controlled=True),
        # an update over the headline batch: what comes back goes on along the residual stream
        _case("norm grad 10v10 x16384", op="norm_grad", rows=16384 * 20, units=20, width=512, type="bf16",
              out="bf16", controlled=True, stream=True),
        # an odd-sized batch of wide rows, columns of a wider array, the first of its network
        _case("norm grad 9v8 x2501 x1000", op="norm_grad", rows=2501 * 17, units=17, width=1000, type="f32",
              out="f16", residual=False, pad=24),
        # queries and keys of the headline batch, by tick and place
        _case("rotary 10v10 x16384", op="rotary", rows=16384 * 20, units=20, heads=8, width=64, pairs=32,
              type="bf16"),
        # the way back of an odd-sized batch whose heads are turned in part, by place alone
        _case("rotary back 9v8 x5003", op="rotary", rows=5003 * 17, units=17, heads=6, width=40, pairs=15,
              axes=2, interleaved=True, inverse=True, joined=False),
        # one tick of a handful of duels
        _case("step 3v3 x16", op="step", rows=16 * 6, units=6, heads=4, key=32, value=32, type="bf16", ends=0.01),
        # one tick of the headline batch, every unit with a memory of its own
        _case("step 10v10 x16384", op="step", rows=16384 * 20, units=20, heads=4, key=32, value=32, type="bf16",
              ends=0.01),
        # an update over 128 ticks of 256 envs, whose episodes end and begin among them
        _case("attention 10v10 x256 x128 ticks", op="attention", rows=256 * 20, units=20, ticks=128, heads=4,
              key=64, value=64, type="bf16", ends=0.015),
        # two units over one long record: as few rows as there can be, and a long way
        _case("attention 1v1 x32768 ticks", op="attention", rows=2, units=2, ticks=32768, heads=4, key=128,
              value=128, type="bf16", ends=0.0002),
        # the way back of an update over 64 ticks
        _case("attention grad 10v10 x256 x64 ticks", op="attention_grad", rows=256 * 20, units=20, ticks=64,
              heads=4, key=64, value=64, type="bf16", ends=0.015),
        # the way back of an odd-sized one in 32 bits, keys and values of different widths
        _case("attention grad 9v8 x37 x100 ticks", op="attention_grad", rows=37 * 17, units=17, ticks=100,
              heads=3, key=48, value=80, type="f32", joined=False, controlled=True, ends=0.015),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    c = dict(BASE)
    c["op"] = rng.choice(["norm", "norm_grad", "rotary", "step", "attention", "attention", "attention_grad",
                          "attention_grad"])
    c["type"] = rng.choice(["f32", "bf16", "bf16", "f16"])
    c["units"] = _spread(rng, 2, 128)
    c["controlled"] = rng.random() < 0.4
    if c["op"] in ("norm", "norm_grad"):
        c["width"] = _spread(rng, 8, 6000)
        c["out"] = rng.choice(["f32", "bf16", "f16", "e4m3"] if c["op"] == "norm" else ["f32", "bf16", "f16"])
        c["residual"], c["stream"] = rng.random() < 0.7, rng.random() < 0.6
        c["pad"] = rng.choice([0, 0, rng.randint(1, 40)])
        envs = _spread(rng, 1, max(1, 130000000 // (c["units"] * (c["width"] + c["pad"]))))
    elif c["op"] == "rotary":
        c["axes"] = rng.choice([1, 2, 3, 3])
        c["heads"], c["width"] = rng.randint(1, 16), _spread(rng, 2 * c["axes"], 256)
        c["pairs"] = rng.choice([c["width"] // 2, rng.randint(c["axes"], c["width"] // 2)])
        c["interleaved"], c["inverse"], c["joined"] = rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.6
        c["first_tick"] = rng.choice([0, 0, _spread(rng, 1000, 10 ** 9)])
        envs = _spread(rng, 1, max(1, 150000000 // (c["units"] * c["heads"] * c["width"])))
    else:
        c["heads"] = rng.randint(1, 8)
        c["key"] = _spread(rng, 4, 128)
        c["value"] = c["key"] if rng.random() < 0.6 else _spread(rng, 4, 128)
        c["joined"], c["state"] = rng.random() < 0.6, rng.random() < 0.7
        per_row = c["heads"] * (c["key"] + c["value"])
        if c["op"] == "step":
            most = 600000000 // (c["units"] * c["heads"] * c["key"] * c["value"])
            c["ends"] = rng.choice([0.0, 0.01, 0.2])
        else:
            c["ticks"] = _spread(rng, 1, 32768 if c["op"] == "attention" else 8192)
            c["units"] = min(c["units"], max(1, 40000000 // (c["ticks"] * per_row)))
            most = min(70000000 // (c["ticks"] * per_row * c["units"]),
                       600000000 // (c["units"] * c["heads"] * c["key"] * c["value"]))
            c["ends"] = rng.choice([0.0, 0.015, 2.0 / c["ticks"], 0.3])
        envs = _spread(rng, 1, max(1, most))
    c["rows"] = envs * c["units"]
    return c


def _learns(c, dev):
    """Bytes [rows]: the first half of every env's units, or None where all of them learn."""
    if not c["controlled"]:
        return None
    return (torch.arange(c["rows"], device=dev) % c["units"] < (c["units"] + 1) // 2).to(torch.uint8)


def prepare(case, seed, device="cuda:0"):
    c, dev = dict(BASE, **case), device
    g = torch.Generator(device=dev).manual_seed(seed)
    R, W, H, T, t = c["rows"], c["width"], c["heads"], c["ticks"], TYPES[c["type"]]

    def uni(*shape):
        return torch.rand(*shape, generator=g, device=dev)

    def normal(*shape, type=torch.float32):
        return torch.randn(*shape, generator=g, device=dev, dtype=type)

    s = {"case": c, "learns": _learns(c, dev), "workspace": None}
    if c["op"] in ("norm", "norm_grad"):
        def rows(n, m, size, type):
            return (size * normal(n, m + c["pad"])).to(type)[:, :m]

        s["weight"] = 1.0 + 0.1 * normal(W)
        if c["op"] == "norm":
            s["x"] = rows(R, W, 1.0, t)
            s["residual"] = rows(R, W, 2.0, t) if c["residual"] else None
            s["sum"] = torch.full((R, W), 0.25, dtype=t, device=dev) if c["residual"] else None
            s["y"] = torch.full((R, W), 0.5, device=dev).to(TYPES[c["out"]])
            s["scale"] = uni(R) if c["out"] == "e4m3" else None
            s["rstd"] = uni(R)
        else:
            s["sum"] = rows(R, W, 2.0, t)
            s["rstd"] = torch.rsqrt(s["sum"].float().square().mean(1) + EPS)
            s["grad_y"] = rows(R, W, 1.0, TYPES[c["out"]])
            s["grad_sum"] = rows(R, W, 0.5, t) if c["stream"] else None
            s["grad_x"] = torch.empty(R, W, dtype=t, device=dev)
            s["grad_weight"] = torch.empty(W, device=dev)
        return s
    E = R // c["units"]
    if c["op"] == "rotary":
        # queries and keys are the first columns of a projection's output, beside as many values
        wide = H * W + (H * W // 2 if c["joined"] else 0)
        s["x"] = normal(R, wide).to(t)[:, :H * W].view(R, H, W)
        s["y"] = torch.full((R, H, W), 0.5, dtype=t, device=dev)
        tick = (c["first_tick"] + torch.randint(0, 300, (E,), generator=g, device=dev)).to(torch.int32)
        where = [tick, 64.0 * uni(R), 64.0 * uni(R)] if c["axes"] != 2 else [64.0 * uni(R), 64.0 * uni(R)]
        left, s["axes"], frequency = c["pairs"], [], []
        for n, position in enumerate(where[:c["axes"]]):
            pairs = left // (c["axes"] - n)
            left -= pairs
            base = 10000.0 if position.dtype == torch.int32 else 100.0
            s["axes"].append((position, pairs))
            frequency.append(base ** (-torch.arange(pairs, device=dev, dtype=torch.float64) / max(pairs, 1)))
        s["frequency"] = torch.cat(frequency)
        return s
    K, V = c["key"], c["value"]
    small = K ** -0.25

    def heads(*lead):
        if c["joined"]:
            x = normal(*lead, H * (2 * K + V))
            x[..., :2 * H * K] *= small
            x = x.to(t)
            return [x[..., :H * K].unflatten(-1, (H, K)), x[..., H * K:2 * H * K].unflatten(-1, (H, K)),
                    x[..., 2 * H * K:].unflatten(-1, (H, V))]
        return [(size * normal(*lead, H, n)).to(t) for size, n in ((small, K), (small, K), (1.0, V))]

    s["scale"] = K ** -0.5
    s["log_decay"] = torch.log1p(-(2.0 ** -(2.0 + torch.arange(H, device=dev) * (6.0 / H))))
    if c["op"] == "step":
        s["q"], s["k"], s["v"] = heads(R)
        s["state"] = normal(R, H, K, V)
        s["fresh"] = (uni(E) < c["ends"]).to(torch.uint8) if c["ends"] else None
        s["out"] = torch.full((R, H, V), 0.5, dtype=t, device=dev)
        return s
    s["q"], s["k"], s["v"] = heads(T, R)
    s["fresh"] = (uni(T, E) < c["ends"]).to(torch.uint8) if c["ends"] else None
    s["state_in"] = normal(R, H, K, V) if c["state"] else None
    if c["op"] == "attention":
        s["state_out"] = torch.full((R, H, K, V), 0.25, device=dev) if c["state"] else None
        s["out"] = torch.full((T, R, H, V), 0.5, dtype=t, device=dev)
    else:
        s["grad_out"] = normal(T, R, H, V).to(t)
        s["grad_state_out"] = 0.1 * normal(R, H, K, V) if c["state"] else None
        s["grad_state_in"] = torch.empty(R, H, K, V, device=dev) if c["state"] else None
        s["grad_q"], s["grad_k"] = (torch.empty(T, R, H, K, dtype=t, device=dev) for _ in range(2))
        s["grad_v"] = torch.empty(T, R, H, V, dtype=t, device=dev)
    return s


def _where_learns(s, new, old, dim=0):
    """`new` for the rows (dimension `dim`) that learn, `old` for the others."""
    if s["learns"] is None or new is None:
        return new
    keep = (s["learns"] != 0).view((1,) * dim + (-1,) + (1,) * (new.dim() - dim - 1))
    return torch.where(keep, new.float(), old.float()).to(new.dtype)


def _plain_norm(s):
    x = s["x"].float()
    out = {}
    if s["residual"] is not None:
        total = (x + s["residual"].float()).to(s["sum"].dtype)
        out["sum"] = _where_learns(s, total, s["sum"])
        x = total.float()
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    out["rstd"] = _where_learns(s, rstd, s["rstd"])
    y = x * rstd[:, None] * s["weight"]
    if s["scale"] is not None:
        scale = (y.abs().amax(1) / LARGEST).clamp(min=SMALLEST_SCALE)
        out["scale"] = _where_learns(s, scale, s["scale"])
        y = y / scale[:, None]
    out["y"] = _where_learns(s, y.to(s["y"].dtype), s["y"])
    return out


def _plain_norm_grad(s):
    h = s["sum"].float() * s["rstd"][:, None]
    gy = _where_learns(s, s["grad_y"].float(), torch.zeros((), device=h.device))
    g = gy * s["weight"]
    gx = s["rstd"][:, None] * (g - h * (g * h).mean(1, keepdim=True))
    if s["grad_sum"] is not None:
        gx = gx + _where_learns(s, s["grad_sum"].float(), torch.zeros((), device=h.device))
    return {"grad_x": gx.to(s["grad_x"].dtype), "grad_weight": (gy * h).sum(0)}


def _turns(s):
    """Angles [rows, pairs] in 64 bits, between -pi and pi: far positions turn often."""
    R, at, parts = s["case"]["rows"], 0, []
    for position, pairs in s["axes"]:
        p = position.double().repeat_interleave(R // position.numel())
        parts.append(p[:, None] * s["frequency"][at:at + pairs])
        at += pairs
    a = torch.cat(parts, 1)
    return a - 2.0 * math.pi * torch.round(a / (2.0 * math.pi))


def _plain_rotary(s):
    c = s["case"]
    P, a = c["pairs"], _turns(s).float()[:, None, :]
    cos, sin = torch.cos(a), torch.sin(a) * (-1.0 if c["inverse"] else 1.0)
    x = s["x"].float()
    if c["interleaved"]:
        u, v = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
        turned = torch.stack((u * cos - v * sin, u * sin + v * cos), -1).flatten(-2)
    else:
        u, v = x[..., :P], x[..., P:2 * P]
        turned = torch.cat((u * cos - v * sin, u * sin + v * cos), -1)
    y = torch.cat((turned, x[..., 2 * P:]), -1).to(s["y"].dtype)
    return {"y": _where_learns(s, y, s["y"])}


def _plain_step(s):
    c = s["case"]
    q, k, v = (s[n].float() for n in ("q", "k", "v"))
    state = s["state"] * torch.exp(s["log_decay"])[None, :, None, None]
    if s["fresh"] is not None:
        state = torch.where(s["fresh"].repeat_interleave(c["units"])[:, None, None, None] != 0, 0.0, state)
    state = state + k[..., :, None] * v[..., None, :]
    out = torch.matmul(q[..., None, :], state)[..., 0, :] * s["scale"]
    # the state is the program's own: it is written where it lies
    s["state"].copy_(_where_learns(s, state, s["state"]))
    return {"out": _where_learns(s, out.to(s["out"].dtype), s["out"]), "state": s["state"]}


CHUNK = 64


def _scan(q, k, v, decay, fresh, units, state, first):
    """sum over s <= t of the same episode of exp(decay (t - s)) (q_t . k_s) v_s, beside what is left of
    `state` (exp(decay (t + first)) q_t state), for q, k, v [T, R, H, *] in 32 bits; and the last tick's
    sum of exp(decay (T - 1 - s)) k_s v_s, with whether `state` is still part of its episode."""
    T, R, H = q.shape[:3]
    n = -(-T // CHUNK)
    dev = q.device

    def chunks(x):
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, 0, 0, n * CHUNK - T))
        return x.permute(1, 2, 0, 3).contiguous().view(R, H, n, CHUNK, x.shape[-1])

    # ticks behind the last one take no time and belong to its episode
    time = torch.arange(n * CHUNK, device=dev).clamp(max=T - 1)
    if fresh is None:
        episode = torch.zeros(R, n * CHUNK, device=dev, dtype=torch.int32)
    else:
        episode = fresh.int().cumsum(0, dtype=torch.int32)[time].t().contiguous().repeat_interleave(units, 0)
    time, episode = time.view(n, CHUNK), episode.view(R, 1, n, CHUNK)
    last, end = episode[..., -1], time[:, -1]
    before = torch.nn.functional.pad(last[..., :-1], (1, 0))
    start = torch.nn.functional.pad(end[:-1], (1, 0), value=-1)
    decay = decay.view(H, 1, 1)

    def left(ticks):
        return torch.exp(decay * ticks.clamp(min=0).float())

    q, k, v = chunks(q), chunks(k), chunks(v)
    within = torch.matmul(q, k.transpose(-1, -2).contiguous())
    age = time[:, :, None] - time[:, None, :]
    within *= torch.exp(decay[..., None] * age.clamp(min=0).float())
    earlier = torch.ones(CHUNK, CHUNK, device=dev, dtype=torch.bool).tril()
    within *= (episode[..., :, None] == episode[..., None, :]) & earlier
    out = torch.matmul(within, v)
    del within
    # what every chunk adds to the state, what lies behind each, and what is read of that
    kept = left(end[:, None] - time) * (episode == last[..., None])
    added = torch.matmul((k * kept[..., None]).transpose(-1, -2).contiguous(), v).flatten(-2)
    to = left(end[:, None] - end[None, :]) * (last[..., :, None] == last[..., None, :])
    to = to * torch.ones(n, n, device=dev).tril()
    behind = torch.matmul(to, added)
    final = behind[:, :, -1].unflatten(-1, (q.shape[-1], v.shape[-1]))
    if n > 1:
        earlier = torch.nn.functional.pad(behind[:, :, :-1], (0, 0, 1, 0)).unflatten(-1, (q.shape[-1], v.shape[-1]))
        weight = left(time - start[:, None]) * (episode == before[..., None])
        out += torch.matmul(q, earlier) * weight[..., None]
    if state is not None:
        weight = left(time + first) * (episode == 0)
        out += torch.matmul(q, state[:, :, None]) * weight[..., None]
    out = out.flatten(2, 3)[:, :, :T].permute(2, 0, 1, 3)
    return out, final, (last[:, :, -1] == 0)[..., None, None]


def _plain_attention(s):
    c = s["case"]
    out, final, still = _scan(s["q"].float(), s["k"].float(), s["v"].float(), s["log_decay"], s["fresh"],
                              c["units"], s["state_in"], 1)
    answer = {"out": _where_learns(s, (out * s["scale"]).to(s["out"].dtype), s["out"], 1)}
    if c["state"]:
        left = torch.exp(s["log_decay"] * float(c["ticks"]))[None, :, None, None]
        final = final + torch.where(still, s["state_in"] * left, 0.0)
        answer["state_out"] = _where_learns(s, final, s["state_out"])
    return answer


def _plain_attention_grad(s):
    c, g, units = s["case"], s["log_decay"], s["case"]["units"]
    q, k, v, go = s["q"].float(), s["k"].float(), s["v"].float(), s["grad_out"].float() * s["scale"]

    def swapped(state):
        return None if state is None else state.transpose(-1, -2).contiguous()

    gq, _, _ = _scan(go, v, k, g, s["fresh"], units, swapped(s["state_in"]), 1)
    # backwards in time an episode begins where, forwards, the next one does
    fresh = s["fresh"]
    if fresh is not None:
        fresh = torch.cat((torch.zeros_like(fresh[:1]), fresh[1:].flip(0)))
    q, k, v, go = (x.flip(0) for x in (q, k, v, go))
    gk, _, _ = _scan(v, go, q, g, fresh, units, swapped(s["grad_state_out"]), 0)
    gv, final, still = _scan(k, q, go, g, fresh, units, s["grad_state_out"], 0)
    zero = torch.zeros((), device=q.device)
    answer = {n: _where_learns(s, x, zero, 1).to(s[n].dtype)
              for n, x in (("grad_q", gq), ("grad_k", gk.flip(0)), ("grad_v", gv.flip(0)))}
    if c["state"]:
        left = torch.exp(g * float(c["ticks"]))[None, :, None, None]
        final = final * torch.exp(g)[None, :, None, None] + torch.where(still, s["grad_state_out"] * left, 0.0)
        if s["fresh"] is not None:
            final = torch.where(s["fresh"][0].repeat_interleave(units)[:, None, None, None] != 0, 0.0, final)
        answer["grad_state_in"] = _where_learns(s, final, zero)
    return answer


def _own(s):
    from paper_2602_01665_amd import binding as B
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        B.tabx_rms_norm(s["x"], s["weight"], EPS, s["y"], s["scale"], s["rstd"], s["residual"], s["sum"],
                        s["learns"])
        return {k: s[k] for k in ("sum", "rstd", "scale", "y") if s[k] is not None}
    if op == "norm_grad":
        if s["workspace"] is None:
            s["workspace"] = torch.empty(B.tabx_rms_norm_workspace(c["rows"], c["width"]), dtype=torch.uint8,
                                         device=s["sum"].device)
        B.tabx_rms_norm_backward(s["sum"], s["weight"], s["rstd"], s["grad_y"], s["grad_sum"], s["grad_x"],
                                 s["grad_weight"], s["workspace"], s["learns"])
        return {k: s[k] for k in ("grad_x", "grad_weight")}
    if op == "rotary":
        B.tabx_rotary(s["x"], s["axes"], s["frequency"], s["y"], c["interleaved"], c["inverse"], s["learns"])
        return {"y": s["y"]}
    if op == "step":
        B.tabx_linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["state"], s["out"],
                                     s["fresh"], s["learns"])
        return {k: s[k] for k in ("out", "state")}
    if s["workspace"] is None:
        s["workspace"] = torch.empty(
            B.tabx_linear_attention_workspace(c["ticks"], c["rows"], c["heads"], c["key"], c["value"]),
            dtype=torch.uint8, device=s["q"].device)
    if op == "attention":
        B.tabx_linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["out"], s["fresh"],
                                s["state_in"], s["state_out"], s["workspace"], s["learns"])
        return {k: s[k] for k in ("out", "state_out") if s[k] is not None}
    B.tabx_linear_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["grad_out"],
                                     s["grad_q"], s["grad_k"], s["grad_v"], s["fresh"], s["state_in"],
                                     s["grad_state_out"], s["grad_state_in"], s["workspace"], s["learns"])
    return {k: s[k] for k in ("grad_q", "grad_k", "grad_v", "grad_state_in") if s[k] is not None}


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "rotary": _plain_rotary, "step": _plain_step,
         "attention": _plain_attention, "attention_grad": _plain_attention_grad}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


def work(case):
    """Bytes: what each input and output holds, of the rows that learn where only those are needed."""
    c = dict(BASE, **case)
    R, W, H, T, b = c["rows"], c["width"], c["heads"], c["ticks"], BYTES[c["type"]]
    n, flags = R, 0
    if c["controlled"]:
        n, flags = R // c["units"] * ((c["units"] + 1) // 2), R
    if c["op"] == "norm":
        per = W * (b * (3 if c["residual"] else 1) + BYTES[c["out"]]) + 4 + (4 if c["out"] == "e4m3" else 0)
        return {"bytes": n * per + 4 * W + flags, "flops": 6 * n * W}
    if c["op"] == "norm_grad":
        per = W * (b * (2 if c["stream"] else 1) + BYTES[c["out"]]) + 4
        return {"bytes": n * per + R * W * b + 8 * W + flags, "flops": 10 * n * W}
    if c["op"] == "rotary":
        where = 4 * (R // c["units"] if c["axes"] != 2 else 0) + 4 * n * (c["axes"] - (c["axes"] != 2))
        return {"bytes": 2 * n * H * W * b + where + 8 * c["pairs"] + flags, "flops": 6 * n * H * c["pairs"]}
    K, V = c["key"], c["value"]
    if c["op"] == "step":
        return {"bytes": n * H * ((2 * K + 2 * V) * b + 8 * K * V) + flags + (R // c["units"] if c["ends"] else 0),
                "flops": 5 * n * H * K * V}
    ends = T * (R // c["units"]) if c["ends"] else 0
    states = n * H * K * V * 4 if c["state"] else 0
    if c["op"] == "attention":
        return {"bytes": T * n * H * (2 * K + 2 * V) * b + 2 * states + ends + flags, "flops": 4 * T * n * H * K * V}
    return {"bytes": T * H * (n * (2 * K + 2 * V) + R * (2 * K + V)) * b + 2 * states + R * H * K * V * 4 * c["state"] + ends + flags,
            "flops": 12 * T * n * H * K * V}


def exact(case, seed, device="cuda:0"):
    s = prepare(case, seed, device)
    c = s["case"]
    R, H, T = c["rows"], c["heads"], c["ticks"]
    on = torch.arange(R, device=device) if s["learns"] is None else s["learns"].nonzero()[:, 0]

    def put(old, new, dim=0):
        """`new`, of the rows that learn, among the `old` ones (a tensor, or a number for all)."""
        if s["learns"] is None:
            return new
        shape = list(new.shape)
        shape[dim] = R
        whole = torch.full(shape, old, dtype=torch.float64, device=device) if isinstance(old, float) else old.double()
        return whole.index_copy(dim, on, new)

    if c["op"] == "norm":
        total = s["x"][on].double()
        out = {}
        if c["residual"]:
            total += s["residual"][on].double()
            out["sum"] = put(s["sum"], total)
            total = total.float().to(s["sum"].dtype).double()     # the norm is that of the sum as it is kept
        rstd = (torch.einsum("rw,rw->r", total, total) / c["width"] + EPS) ** -0.5
        out["rstd"] = put(s["rstd"], rstd)
        y = total.mul_(s["weight"].double()).mul_(rstd[:, None])
        if c["out"] == "e4m3":
            scale = torch.maximum(y.max(1).values, -y.min(1).values) * (1.0 / LARGEST)
            scale = scale.clamp(min=SMALLEST_SCALE)
            out["scale"] = put(s["scale"], scale)
            # eight bits: four digits of the value, three of them behind the point, 2^-9 at the least
            y /= scale[:, None]
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
            y = torch.round(y / step) * step
        out["y"] = put(s["y"], y)
        return out
    if c["op"] == "norm_grad":
        rstd, W = s["rstd"][on].double()[:, None], c["width"]
        x, gy = s["sum"][on].double(), s["grad_y"][on].double()
        gw = torch.einsum("rw,rw->w", x * rstd, gy)
        gy = gy * s["weight"].double()
        dot = torch.einsum("rw,rw->r", x, gy)[:, None]
        gx = rstd * gy - x * (rstd ** 3 * dot / W)
        if c["stream"]:
            gx += s["grad_sum"][on].double()
        return {"grad_x": put(0.0, gx), "grad_weight": gw}
    if c["op"] == "rotary":
        x = s["x"][on].double()
        P, at, angle = c["pairs"], 0, torch.empty(len(on), c["pairs"], dtype=torch.float64, device=device)
        for position, pairs in s["axes"]:
            p = position.double()[on // (R // position.numel())]
            angle[:, at:at + pairs] = torch.outer(p, torch.ones(pairs, dtype=torch.float64, device=device))
            at += pairs
        angle *= s["frequency"]
        turn = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)[:, None]
        if c["interleaved"]:
            z = torch.view_as_complex(x[..., :2 * P].reshape(len(on), H, P, 2).contiguous()) * turn
            x[..., :2 * P] = torch.view_as_real(z).reshape(len(on), H, 2 * P)
        else:
            z = torch.complex(x[..., :P].contiguous(), x[..., P:2 * P].contiguous()) * turn
            x[..., :P], x[..., P:2 * P] = z.real, z.imag
        return {"y": put(s["y"], x)}
    gamma = torch.exp(s["log_decay"].double())[:, None, None]
    env = on // c["units"]
    if c["op"] == "step":
        # a part of the rows at a time: the states are many
        whole, states = torch.empty(len(on), H, c["value"], dtype=torch.float64, device=device), []
        for b in range(0, len(on), 65536):
            r = on[b:b + 65536]
            state = s["state"][r].double()
            if s["fresh"] is not None:
                state[s["fresh"][r // c["units"]] != 0] = 0.0
            state.mul_(gamma).addcmul_(s["k"][r].double()[..., None], s["v"][r].double()[..., None, :])
            whole[b:b + 65536] = (s["q"][r].double()[..., None] * state).sum(-2) * s["scale"]
            states.append(state)
        state = torch.cat(states)
        if s["learns"] is not None:
            state = put(s["state"], state)
        return {"out": put(s["out"], whole), "state": state}
    K, V = c["key"], c["value"]

    def at(x, t):
        return x[t][on].double()

    def forgets(t):
        return None if s["fresh"] is None else (s["fresh"][t][env] != 0)[:, None, None, None]

    def forward(visit):
        """Tick after tick: the state forgets, fades, takes the tick in; then it is looked at."""
        state = torch.zeros(len(on), H, K, V, dtype=torch.float64, device=device)
        if c["state"]:
            state += s["state_in"][on]
        for t in range(T):
            if s["fresh"] is not None:
                state.masked_fill_(forgets(t), 0.0)
            state.mul_(gamma).addcmul_(at(s["k"], t)[..., None], at(s["v"], t)[..., None, :])
            visit(t, state)
        return state

    if c["op"] == "attention":
        out = torch.empty(T, len(on), H, V, dtype=torch.float64, device=device)

        def read(t, state):
            torch.matmul(at(s["q"], t)[..., None, :], state, out=out[t].unsqueeze(-2)).mul_(s["scale"])

        final = forward(read)
        answer = {"out": put(s["out"], out, 1)}
        if c["state"]:
            answer["state_out"] = put(s["state_out"], final)
        return answer
    gq, gk = (torch.empty(T, len(on), H, K, dtype=torch.float64, device=device) for _ in range(2))
    gv = torch.empty(T, len(on), H, V, dtype=torch.float64, device=device)

    def to_q(t, state):
        torch.matmul(state, at(s["grad_out"], t)[..., None], out=gq[t].unsqueeze(-1)).mul_(s["scale"])

    forward(to_q)
    back = torch.zeros(len(on), H, K, V, dtype=torch.float64, device=device)
    if c["state"]:
        back += s["grad_state_out"][on]
    for t in range(T - 1, -1, -1):
        back.addcmul_(at(s["q"], t)[..., None], at(s["grad_out"], t)[..., None, :], value=s["scale"])
        torch.matmul(back, at(s["v"], t)[..., None], out=gk[t].unsqueeze(-1))
        torch.matmul(at(s["k"], t)[..., None, :], back, out=gv[t].unsqueeze(-2))
        back.mul_(gamma)
        if s["fresh"] is not None:
            back.masked_fill_(forgets(t), 0.0)
    answer = {n: put(0.0, x, 1) for n, x in (("grad_q", gq), ("grad_k", gk), ("grad_v", gv))}
    if c["state"]:
        answer["grad_state_in"] = put(0.0, back)
    return answer
