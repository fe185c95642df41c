"""The calls of a unit's memory as a training program makes them: a rollout tick by tick with a network of them, the
same ticks at once, the way back; on streams, in graphs and on parts of a batch."""
import pytest
import torch

from tests import memory_reference as M

pytestmark = pytest.mark.gpu
F64 = torch.float64
EPS = 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def batch(B, E=24, steps=9, **kw):
    from paper_2602_01665_amd import inputs as I
    w = I.WORKLOADS["c2_4096env_5v5"]
    env = B.TabxEnv(I.make_params(w, E, max_steps=steps), I.make_scenario(w, E), **kw)
    env.reset()
    env.observe()
    return w, env


class Block:
    """Norm behind a residual, queries, keys and values in one product, turned by tick and place, a memory, a product back
    into the stream."""

    def __init__(self, D, W, H, K, V, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.W, self.H, self.K, self.V = W, H, K, V
        self.inward = (torch.randn(D, W, generator=g) * D ** -0.5 * 0.1).cuda()
        self.weight = (1.0 + 0.1 * torch.randn(W, generator=g)).cuda()
        self.project = (torch.randn(W, H * (2 * K + V), generator=g) * W ** -0.5).cuda()
        self.back = (torch.randn(H * V, W, generator=g) * (H * V) ** -0.5).cuda()
        self.pairs = (K // 2 - 2 * (K // 6), K // 6, K // 6)
        self.frequency = torch.cat([50.0 ** (-torch.arange(n, dtype=F64) / n) for n in self.pairs]).cuda()
        self.decay = M.decays(H).cuda()
        self.scale = K ** -0.5

    def split(self, qkv):
        n = self.H * self.K
        return (qkv[..., :2 * n].unflatten(-1, (2 * self.H, self.K)), qkv[..., 2 * n:].unflatten(-1, (self.H, self.V)))


def plain_block(b, x, residual, weight, project, back, places, fresh, state):
    """The block over ticks from elementary operations: x, residual [T, E, N, W], places (t [T, E], x, y [T, E, N])."""
    T, E, N, W = x.shape
    s = x + residual
    y = s / torch.sqrt((s * s).mean(-1, keepdim=True) + EPS) * weight
    qkv = y @ project
    qk, v = qkv[..., :2 * b.H * b.K].unflatten(-1, (2 * b.H, b.K)), qkv[..., 2 * b.H * b.K:].unflatten(-1, (b.H, b.V))
    at, parts = 0, []
    for p, n in zip(places, b.pairs):
        p = p.double()[..., None].expand(T, E, N) if p.dim() == 2 else p.double()
        parts.append(p[..., None] * b.frequency.to(p.device)[at:at + n])
        at += n
    a = torch.cat(parts, -1)[..., None, :].to(s.dtype)
    P = a.shape[-1]
    u, w = qk[..., :P], qk[..., P:2 * P]
    qk = torch.cat((u * torch.cos(a) - w * torch.sin(a), u * torch.sin(a) + w * torch.cos(a), qk[..., 2 * P:]), -1)
    q, k = qk[..., :b.H, :], qk[..., b.H:, :]
    gamma = torch.exp(b.decay.to(s.dtype).to(s.device))[:, None, None]
    outs = []
    for t in range(T):
        state = torch.where(fresh[t][:, None, None, None, None] != 0, torch.zeros((), dtype=s.dtype, device=s.device), state * gamma)
        state = state + k[t][..., :, None] * v[t][..., None, :]
        outs.append((q[t][..., :, None] * state).sum(-2) * b.scale)
    out = torch.stack(outs)
    return s + out.flatten(-2) @ back, state


def test_a_rollout_with_a_memory_and_its_update(B):
    """Twenty ticks whose episodes end at different times: the steps, the ticks at once, and the gradients of the weights
    against autograd of the plain block in 64 bits."""
    w, env = batch(B, steps=7)
    E, N, D, T = env.E, env.N, env.D, 20
    b = Block(D, 48, 2, 12, 16)
    g = torch.Generator().manual_seed(1)
    state = torch.zeros(E, N, b.H, b.K, b.V, device="cuda")
    env.dones.zero_()
    rec = {n: [] for n in ("x", "res", "t", "px", "py", "fresh", "sum", "rstd", "qk", "v", "out", "stream")}
    for tick in range(T):
        x = env.obs @ b.inward
        res = torch.randn(E, N, b.W, generator=g).cuda()
        total, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(E, N, device="cuda")
        B.tabx_rms_norm(x, b.weight, EPS, y, None, rstd, res, total)
        qk, v = b.split(y @ b.project)
        turned = torch.empty(E, N, 2 * b.H, b.K, device="cuda")
        env.rotate(qk, b.pairs, b.frequency, turned)
        out = torch.empty(E, N, b.H, b.V, device="cuda")
        env.remember(turned[..., :b.H, :], turned[..., b.H:, :], v, b.decay, b.scale, state, out)
        stream = total + out.flatten(-2) @ b.back
        for n, t in (("x", x), ("res", res), ("t", env.st["t"]), ("px", env.st["x"].view(E, N)), ("py", env.st["y"].view(E, N)),
                     ("fresh", env.dones), ("sum", total), ("rstd", rstd), ("qk", turned), ("v", v), ("out", out), ("stream", stream)):
            rec[n].append(t.clone())
        env.step_observe(torch.randint(0, 8, (E, N), generator=g).to(torch.uint8).cuda())
    r = {n: torch.stack(t) for n, t in rec.items()}
    assert 0 < int(r["fresh"].sum()) < T * E and int(r["t"].max()) > 2
    # the same in 64 bits, with its graph
    leaves = {n: t.double().requires_grad_() for n, t in (("x", r["x"]), ("weight", b.weight), ("project", b.project), ("back", b.back))}
    places = (r["t"], r["px"], r["py"])
    zero = torch.zeros(E, N, b.H, b.K, b.V, dtype=F64, device="cuda")
    want, after = plain_block(b, leaves["x"], r["res"].double(), leaves["weight"], leaves["project"], leaves["back"], places, r["fresh"], zero)
    size = float(want.abs().max())
    # products of 32 bits of up to a hundred terms, twenty ticks of sums: some 200 roundings of the largest value
    close = 400 * M.U * size
    assert float((r["stream"].double() - want).abs().max()) < close and float((state.double() - after).abs().max()) < 400 * M.U * float(after.abs().max())
    # all ticks at once
    out, last = torch.empty_like(r["out"]), torch.empty_like(state)
    q, k = r["qk"][..., :b.H, :], r["qk"][..., b.H:, :]
    ws = torch.empty(B.tabx_linear_attention_workspace(T, E * N, b.H, b.K, b.V), dtype=torch.uint8, device="cuda")
    B.tabx_linear_attention(q, k, r["v"], b.decay, b.scale, out, r["fresh"], None, last, ws)
    assert float((out - r["out"]).abs().max()) < close and float((last - state).abs().max()) < 400 * M.U * float(after.abs().max())
    # the way back, call by call
    gs = torch.randn(want.shape, generator=g).cuda()
    (want * gs.double()).sum().backward()
    g_out = (gs @ b.back.t()).unflatten(-1, (b.H, b.V))
    g_back = out.flatten(-2).flatten(0, -2).t() @ gs.flatten(0, -2)
    g_qk, g_v = torch.empty_like(r["qk"]), torch.empty_like(r["v"].contiguous())
    B.tabx_linear_attention_backward(q, k, r["v"], b.decay, b.scale, g_out, g_qk[..., :b.H, :], g_qk[..., b.H:, :], g_v, r["fresh"],
                                     workspace=ws)
    axes = [(r["t"], b.pairs[0]), (r["px"], b.pairs[1]), (r["py"], b.pairs[2])]
    B.tabx_rotary(g_qk, axes, b.frequency, g_qk, False, True)
    g_qkv = torch.cat((g_qk.flatten(-2), g_v.flatten(-2)), -1)
    g_y = g_qkv @ b.project.t()
    y = r["sum"] * r["rstd"][..., None] * b.weight
    g_project = y.flatten(0, -2).t() @ g_qkv.flatten(0, -2)
    g_x, g_weight = torch.empty_like(r["x"]), torch.empty_like(b.weight)
    ws2 = torch.empty(B.tabx_rms_norm_workspace(T * E * N, b.W), dtype=torch.uint8, device="cuda")
    B.tabx_rms_norm_backward(r["sum"], b.weight, r["rstd"], g_y, gs, g_x, g_weight, ws2)
    for name, got in (("x", g_x), ("weight", g_weight), ("project", g_project), ("back", g_back)):
        value = leaves[name].grad
        # sums of thousands of terms and chains of four products: some 4000 roundings of the largest value
        assert float((got.double() - value).abs().max()) < 4000 * M.U * float(value.abs().max()), name


def inputs(seed, T, R, H, K, V, dtype=torch.float32):
    g = torch.Generator("cuda").manual_seed(seed)
    q, k = (torch.randn(T, R, H, K, generator=g, device="cuda").to(dtype) for _ in range(2))
    v, go = (torch.randn(T, R, H, V, generator=g, device="cuda").to(dtype) for _ in range(2))
    fresh = (torch.rand(T, R, generator=g, device="cuda") < 0.05).to(torch.uint8)
    return q, k, v, go, fresh, torch.randn(R, H, K, V, generator=g, device="cuda")


class Calls:
    """All calls on buffers of their own; `fill` puts in other values."""

    def __init__(self, B, T, R, H, K, V, dtype):
        self.B, self.shape, self.dtype = B, (T, R, H, K, V), dtype
        self.q, self.k, self.v, self.go, self.fresh, self.s0 = inputs(0, T, R, H, K, V, dtype)
        self.decay = M.decays(H).cuda()
        self.out, self.after = torch.empty_like(self.v), torch.empty_like(self.s0)
        self.gq, self.gk, self.gv, self.gs = (torch.empty_like(t) for t in (self.q, self.k, self.v, self.s0))
        self.ws = torch.empty(B.tabx_linear_attention_workspace(T, R, H, K, V), dtype=torch.uint8, device="cuda")
        self.state, self.one = torch.empty_like(self.s0), torch.empty_like(self.v[0])
        self.x, self.res = torch.empty(T * R, H * V, device="cuda"), torch.empty(T * R, H * V, device="cuda")
        self.y, self.sum = torch.empty_like(self.x).to(torch.float8_e4m3fn), torch.empty_like(self.x)
        self.scale, self.rstd = torch.empty(T * R, device="cuda"), torch.empty(T * R, device="cuda")
        self.gx, self.gw = torch.empty_like(self.x), torch.empty(H * V, device="cuda")
        self.ws2 = torch.empty(B.tabx_rms_norm_workspace(T * R, H * V), dtype=torch.uint8, device="cuda")
        self.t = torch.empty(T * R, dtype=torch.int32, device="cuda")
        self.frequency = torch.ones(K // 2, dtype=F64, device="cuda")
        self.turned = torch.empty_like(self.q)
        self.fill(1)

    def fill(self, seed):
        for mine, new in zip((self.q, self.k, self.v, self.go, self.fresh, self.s0), inputs(seed, *self.shape, self.dtype)):
            mine.copy_(new)
        g = torch.Generator("cuda").manual_seed(seed)
        self.x.normal_(generator=g)
        self.res.normal_(generator=g)
        self.t.random_(0, 1000, generator=g)

    def run(self, stream=None):
        B, kw = self.B, dict(stream=stream)
        B.tabx_rotary(self.q, [(self.t, self.shape[3] // 2)], self.frequency, self.turned, **kw)
        B.tabx_linear_attention(self.turned, self.k, self.v, self.decay, 0.5, self.out, self.fresh, self.s0, self.after, self.ws, **kw)
        B.tabx_linear_attention_backward(self.turned, self.k, self.v, self.decay, 0.5, self.go, self.gq, self.gk, self.gv, self.fresh, self.s0,
                                         self.after, self.gs, self.ws, **kw)
        B.tabx_linear_attention_step(self.q[0], self.k[0], self.v[0], self.decay, 0.5, self.after, self.one, self.fresh[0], **kw)
        B.tabx_rms_norm(self.x, None, EPS, self.y, self.scale, self.rstd, self.res, self.sum, **kw)
        B.tabx_rms_norm_backward(self.sum, None, self.rstd, self.res, self.x, self.gx, self.gw, self.ws2, **kw)

    def results(self):
        return [t.clone() for t in (self.turned, self.out, self.after, self.gq, self.gk, self.gv, self.gs, self.one, self.y.view(torch.uint8),
                                    self.sum, self.scale, self.rstd, self.gx, self.gw)]


SHAPES = [(70, 24, 2, 32, 32, torch.bfloat16), (600, 2, 2, 16, 24, torch.float32), (40, 6, 1, 128, 96, torch.float16)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_captured_and_replayed(B, shape):
    """A graph's replays with other inputs, with eager work and graphs of autograd between them, give what eager calls do."""
    calls = Calls(B, *shape)
    leaf = calls.s0.clone().requires_grad_()
    alive = (leaf * 2.0).sum()                                 # an eager graph that lives through the capture
    eager = []
    for seed in (2, 3, 4):
        calls.fill(seed)
        calls.run()
        eager.append(calls.results())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls.run()
    for turn in range(2):
        for seed, want in zip((2, 3, 4), eager):
            calls.fill(seed)
            graph.replay()
            torch.cuda.synchronize()
            for n, (a, b) in enumerate(zip(calls.results(), want)):
                assert torch.equal(a, b), (turn, seed, n)
            (torch.ones(1000, device="cuda") * turn).sum().item()
    alive.backward()
    assert (leaf.grad == 2.0).all()


def test_two_graphs_at_once_with_a_workspace_each(B):
    a, b = Calls(B, 600, 2, 2, 16, 24, torch.float32), Calls(B, 500, 1, 3, 64, 64, torch.bfloat16)
    want = []
    for c in (a, b):
        c.run()
        want.append(c.results())
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for c in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        graphs.append(graph)
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for c, w in zip((a, b), want):
            for x, y in zip(c.results(), w):
                assert torch.equal(x, y)


def test_on_another_stream(B):
    c = Calls(B, 70, 24, 2, 32, 32, torch.bfloat16)
    c.run()
    want = c.results()
    s = torch.cuda.Stream()
    for t in (c.out, c.after, c.gq, c.sum, c.turned):
        t.zero_()
    torch.cuda.synchronize()
    c.run(s)
    s.synchronize()
    for a, b in zip(c.results(), want):
        assert torch.equal(a, b)


def test_parts_of_a_batch_compute_what_the_whole_would(B):
    w, env = batch(B, E=20, steps=5)
    E, N, H, K, V = env.E, env.N, 2, 12, 8
    g = torch.Generator("cuda").manual_seed(3)
    decay, freq = M.decays(H).cuda(), torch.ones(6, dtype=F64, device="cuda")
    whole, split = torch.zeros(E, N, H, K, V, device="cuda"), torch.zeros(E, N, H, K, V, device="cuda")
    for tick in range(8):
        x, v = torch.randn(E, N, H, K, generator=g, device="cuda"), torch.randn(E, N, H, V, generator=g, device="cuda")
        y, z = torch.empty_like(x), torch.empty_like(x)
        o, p = torch.empty_like(v), torch.empty_like(v)
        env.rotate(x, (2, 2, 2), freq, y)
        env.remember(y, x, v, decay, 0.3, whole, o)
        for part in env.parts(3):
            c = slice(part.first_env, part.first_env + part.E)
            part.rotate(x[c], (2, 2, 2), freq, z[c])
            part.remember(z[c], x[c], v[c], decay, 0.3, split[c], p[c])
        assert torch.equal(y, z) and torch.equal(o, p) and torch.equal(whole, split)
        env.step_observe(torch.randint(0, 8, (E, N), generator=g, device="cuda").to(torch.uint8))
    assert int(env.st["t"].max()) < 8


def test_a_graph_of_autograd_is_told_what_was_written(B):
    T, R, H, K, V = 4, 3, 1, 8, 8
    q, k, v, go, fresh, s0 = inputs(5, T, R, H, K, V)
    leaf = torch.ones_like(s0, requires_grad=True)
    loss = (leaf * s0).sum()                                   # its way back needs s0 as it is
    B.tabx_linear_attention_step(q[0], k[0], v[0], M.decays(H).cuda(), 1.0, s0, torch.empty_like(v[0]))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    before = [t._version for t in (q, v, go)]
    out = torch.empty_like(v)
    B.tabx_linear_attention(q, k, v, M.decays(H).cuda(), 1.0, out, fresh)
    assert out._version == 1 and [t._version for t in (q, v, go)] == before


def test_a_stream_of_another_device_is_refused(B):
    class Elsewhere:
        device_index, device, cuda_stream = 1, "cuda:1", 0
    q = torch.zeros(2, 1, 8, device="cuda")
    with pytest.raises(B.TabxError, match="stream is on"):
        B.tabx_linear_attention_step(q, q, q, torch.zeros(1, device="cuda"), 1.0, torch.zeros(2, 1, 8, 8, device="cuda"), q.clone(), stream=Elsewhere())
