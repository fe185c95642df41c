"""The learner's calls as a training program makes them: a rollout of observations, layer norms,
draws and ticks, the way back through both layer norms, and the same calls in captured graphs and on
other streams (needs an MI355X)."""
import numpy as np
import pytest
import torch

from paper_2602_01665_amd import inputs as I
from tests import learner_reference as R

pytestmark = pytest.mark.gpu
DEV, EPS = "cuda:0", 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_2602_01665_amd import binding
    return binding


def _env(B, name, E, **over):
    w = I.WORKLOADS[name]
    p = I.make_params(w, E, **over)
    env = B.TabxEnv(p, I.make_scenario(w, over.get("num_levels", E)))
    env.reset()
    env.observe()
    return env


class _Net:
    """Observation -> norm -> tanh(linear) -> norm -> nine columns: eight logits and a value."""

    def __init__(self, B, width, hidden, rows, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.B, self.hidden = B, hidden
        self.p = {"w0": 1 + 0.1 * n(width), "b0": 0.1 * n(width), "m1": n(width, hidden) / width ** 0.5,
                  "w1": 1 + 0.1 * n(hidden), "b1": 0.1 * n(hidden), "m2": n(hidden, 9) / hidden ** 0.5}
        e = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
        self.y0, self.y1, self.out = e(rows, width), e(rows, hidden), e(rows, 9)
        self.stats = [e(rows) for _ in range(4)]
        self.ws = [torch.empty(B.tabx_layer_norm_workspace(rows, w), dtype=torch.uint8, device=DEV) for w in (width, hidden)]

    def forward(self, x, on):
        p, s = self.p, self.stats
        self.B.tabx_layer_norm(x, p["w0"], p["b0"], EPS, self.y0, s[0], s[1], on)
        self.h = torch.tanh(self.y0 @ p["m1"])
        self.B.tabx_layer_norm(self.h, p["w1"], p["b1"], EPS, self.y1, s[2], s[3], on)
        torch.mm(self.y1, p["m2"], out=self.out)
        return self.out[:, :8]

    def backward(self, x, on, g_out):
        p, s = self.p, self.stats
        g = {k: torch.empty_like(v) for k, v in p.items()}
        g["m2"] = self.y1.t() @ g_out
        gy1, gh = g_out @ p["m2"].t(), torch.empty_like(self.h)
        self.B.tabx_layer_norm_backward(self.h, p["w1"], s[2], s[3], gy1, gh, g["w1"], g["b1"], self.ws[1], on)
        gz = gh * (1 - self.h * self.h)
        g["m1"] = self.y0.t() @ gz
        gy0 = gz @ p["m1"].t()
        self.B.tabx_layer_norm_backward(x, p["w0"], s[0], s[1], gy0, None, g["w0"], g["b0"], self.ws[0], on)
        return g


def _plain_loss(p, x, on, actions, amask, adv, coef, dtype):
    """The loss of one update in plain tensor operations of `dtype`, on the CPU."""
    q = {k: v.detach().cpu().to(dtype).requires_grad_() for k, v in p.items()}

    def norm(z, w, b):
        c = z - z.mean(1, keepdim=True)
        return c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * w + b

    h = torch.tanh(norm(x.cpu().to(dtype), q["w0"], q["b0"]) @ q["m1"])
    l = (norm(h, q["w1"], q["b1"]) @ q["m2"])[:, :8].clone()
    l = torch.where((amask.cpu() == 0)[:, None] & (torch.arange(8) == 5), torch.tensor(-1e30, dtype=dtype), l)
    lp = torch.log_softmax(l, 1)
    ent = -(lp.exp() * lp).sum(1)
    taken = lp.gather(1, actions.cpu().long()[:, None])[:, 0]
    keep = on.cpu().to(dtype)
    loss = (-(adv.cpu().to(dtype) * taken) * keep).sum() - coef * (ent * keep).sum()
    loss.backward()
    return {k: v.grad for k, v in q.items()}


def test_rollout_and_update(B):
    """Twenty ticks played by the network on one side and the scripted policy on the other; every
    draw is the one that 64 bits make of the same logits.  Then an update on the last tick's rows:
    the gradients are off from 64 bits by no more than a plain 32-bit chain is, which makes roundings
    of the same sizes in the same places but adds in another order (a factor of four for that)."""
    env = _env(B, "c2_4096env_5v5", 37, max_steps=9)
    E, N, D = env.E, env.N, env.D
    team = env.sc["team"].view(E, N)
    ours, theirs = (1 - team).contiguous(), team
    policy = I.policy("medium", seed=3)
    env.prime_scripted(policy, theirs)
    net = _Net(B, D, 64, E * N, 1)
    g = torch.Generator(device=DEV).manual_seed(5)
    actions = torch.zeros(E, N, dtype=torch.uint8, device=DEV)
    lp = torch.zeros(E, N, device=DEV)
    how = B.TabxSampling(0.9, 6, 0.95, 0.01)
    ended, on = 0, ours.view(-1)
    for t in range(20):
        x = env.obs.view(E * N, D)
        logits = net.forward(x, on)
        u = torch.rand(E * N, generator=g, device=DEV)
        before, mask = actions.clone(), env.amask.clone()
        env.sample_actions(logits, how, u, actions, lp, ours)
        want = before.view(-1).cpu().numpy().copy()
        rows = R.allowed(R.f64(logits), mask.view(-1).cpu().numpy())
        for r in np.nonzero(on.cpu().numpy())[0]:
            c = R.choose(rows[r], 0.9, 6, 0.95, 0.01, float(u[r]))
            want[r] = 0 if c is None else c
        assert np.array_equal(actions.view(-1).cpu().numpy(), want), t
        kept = (x.clone(), mask, actions.view(-1).clone())
        env.scripted_step_observe(policy, theirs, actions)
        ended += int(env.dones.sum())
    assert ended >= E                              # episodes ended on the way
    x, mask, acts = kept
    net.forward(x, on)
    adv, coef = torch.randn(E * N, generator=g, device=DEV), 0.01
    lp, ent = torch.zeros(E * N, device=DEV), torch.zeros(E * N, device=DEV)
    B.tabx_action_log_prob(net.out[:, :8], acts, 1.0, lp, ent, mask, on)
    g_out = torch.zeros(E * N, 9, device=DEV)
    B.tabx_action_log_prob_backward(net.out[:, :8], acts, 1.0, -adv, torch.full_like(adv, -coef), g_out[:, :8], mask, on)
    got = net.backward(x, on, g_out)
    exact = _plain_loss(net.p, x, on, acts, mask.view(-1), adv, coef, torch.float64)
    plain = _plain_loss(net.p, x, on, acts, mask.view(-1), adv, coef, torch.float32)
    for k, v in exact.items():
        size = float(v.norm())
        off, other = float((got[k].cpu().double() - v).norm()), float((plain[k].double() - v).norm())
        print("[gpu]", k, "off", off / size, "plain", other / size, flush=True)
        assert off <= 4 * other + 64 * R.U * size, k


def test_between_the_ends_pytorch_differentiates(B):
    """The rows' layer norm and the log-probabilities at the ends, a network of PyTorch's between
    them: its graph is entered with the logits' gradient and left with the rows'.  Held to 64 bits
    as the update above."""
    rows, width, dtype = 300, 176, torch.float32
    g = torch.Generator(device=DEV).manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    p = {"w0": 1 + 0.1 * n(width), "b0": 0.1 * n(width), "m1": n(width, 9) / width ** 0.5}
    x, on = 3.0 * n(rows, width), (n(rows) > 0).to(torch.uint8)
    acts = torch.randint(0, 8, (rows,), generator=g, device=DEV).to(torch.uint8)
    adv, coef = n(rows), 0.02
    y, mean, rstd = torch.zeros(rows, width, device=DEV), torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
    B.tabx_layer_norm(x, p["w0"], p["b0"], EPS, y, mean, rstd, on)
    y.requires_grad_()
    m1 = p["m1"].clone().requires_grad_()
    logits = torch.tanh(y @ m1)[:, :8]
    grad_logits = torch.empty(rows, 8, device=DEV)
    B.tabx_action_log_prob_backward(logits, acts, 1.0, -adv, torch.full_like(adv, -coef), grad_logits, None, on)
    logits.backward(grad_logits)
    got = {"m1": m1.grad, "w0": torch.empty(width, device=DEV), "b0": torch.empty(width, device=DEV)}
    ws = torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)
    B.tabx_layer_norm_backward(x, p["w0"], mean, rstd, y.grad, None, got["w0"], got["b0"], ws, on)
    want = []
    for t in (torch.float64, torch.float32):
        q = {k: v.detach().cpu().to(t).requires_grad_() for k, v in p.items()}
        z = x.cpu().to(t)
        c = z - z.mean(1, keepdim=True)
        h = c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * q["w0"] + q["b0"]
        h = torch.where(on.cpu()[:, None] != 0, h, torch.zeros((), dtype=t))
        lp = torch.log_softmax(torch.tanh(h @ q["m1"])[:, :8], 1)
        keep = on.cpu().to(t)
        taken = lp.gather(1, acts.cpu().long()[:, None])[:, 0]
        ((-(adv.cpu().to(t) * taken) + coef * (lp.exp() * lp).sum(1)) * keep).sum().backward()
        want.append({k: v.grad for k, v in q.items()})
    for k, v in want[0].items():
        off, other = float((got[k].cpu().double() - v).norm()), float((want[1][k].double() - v).norm())
        assert off <= 4 * other + 64 * R.U * float(v.norm()), (k, off, other)
    assert y.dtype is dtype


def test_observations_of_the_learning_side_alone(B):
    """norm_obs on the environment's own rows: the other side's are left as they were."""
    env = _env(B, "c3_16384env_10v10", 50)
    E, N, D = env.E, env.N, env.D
    ours = (1 - env.sc["team"]).view(E, N)
    y = torch.full((E, N, D), 4.0, dtype=torch.bfloat16, device=DEV)
    mean, rstd = torch.zeros(E, N, device=DEV), torch.zeros(E, N, device=DEV)
    w, b = torch.rand(D, device=DEV), torch.rand(D, device=DEV)
    env.norm_obs(w, b, EPS, y, mean, rstd, ours)
    want, _, _, bound, _, _ = R.norm(R.f64(env.obs).reshape(E * N, D), R.f64(w), R.f64(b), float(np.float32(EPS)), y.dtype)
    on = ours.view(-1).cpu().numpy() != 0
    R.near(R.f64(y).reshape(E * N, D)[on], want[on], bound[on], "rows")
    assert bool((y.view(E * N, D)[torch.from_numpy(~on).to(DEV)] == 4).all())


def test_levels_that_were_drawn_are_played(B):
    L, E = 13, 300
    env = _env(B, "c2_4096env_5v5", E, num_levels=L, level_seed=3)
    scores = torch.arange(L, device=DEV, dtype=torch.float32) / 4
    u = torch.rand(E, device=DEV)
    some = (torch.arange(E, device=DEV) % 3 != 0).to(torch.uint8)
    before = env.st["next_level"].clone()
    env.sample_levels(scores, B.TabxSampling(1.0, 5), u, None, some)
    drawn = env.st["next_level"].clone()
    assert torch.equal(drawn[some == 0], before[some == 0])
    assert int(drawn[some != 0].min()) >= L - 5 and len(torch.unique(drawn[some != 0])) == 5
    env.reset()
    assert torch.equal(env.st["level"], drawn)


def _calls(B, s):
    """Every learner's call once, on the tensors of s."""
    B.tabx_layer_norm(s["x"], s["w"], s["b"], EPS, s["y"], s["mean"], s["rstd"], s["on"])
    B.tabx_layer_norm_backward(s["x"], s["w"], s["mean"], s["rstd"], s["gy"], s["gx"], s["gw"], s["gb"], s["ws"], s["on"])
    B.tabx_sample_actions(s["logits"], s["how"], s["u"], s["actions"], s["lp"], s["mask"], s["on"])
    B.tabx_action_log_prob(s["logits"], s["actions"], 0.7, s["lp2"], s["ent"], s["mask"], s["on"])
    B.tabx_action_log_prob_backward(s["logits"], s["actions"], 0.7, s["lp2"], s["ent"], s["gl"], s["mask"], s["on"])
    B.tabx_sample_levels(s["scores"], s["how"], s["u"], s["levels"], None, s["on"])


OUTPUTS = ("y", "mean", "rstd", "gx", "gw", "gb", "actions", "lp", "lp2", "ent", "gl", "levels")
INPUTS = ("x", "gy", "logits", "u", "mask", "on", "scores")


def _state(B, seed, rows=3000, width=314):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    bits = lambda: (n(rows) > 0).to(torch.uint8)  # noqa: E731
    s = {"x": n(rows, width), "gy": n(rows, width), "logits": n(rows, 9)[:, :8], "u": torch.rand(rows, generator=g, device=DEV),
         "mask": bits(), "on": bits(), "scores": n(2000), "w": 1 + 0.1 * torch.ones(width, device=DEV), "b": torch.zeros(width, device=DEV),
         "how": B.TabxSampling(0.7, 5, 0.9, 0.01), "ws": torch.empty(B.tabx_layer_norm_workspace(rows, width), dtype=torch.uint8, device=DEV)}
    z = lambda *q: torch.zeros(*q, device=DEV)  # noqa: E731
    s.update(y=z(rows, width).half(), mean=z(rows), rstd=z(rows), gx=z(rows, width), gw=z(width), gb=z(width),
             actions=z(rows).to(torch.uint8), lp=z(rows), lp2=z(rows), ent=z(rows), gl=z(rows, 8), levels=z(rows).int())
    return s


def test_captured_graph(B):
    """Two graphs with a workspace each, replayed several times on new inputs, with eager work in
    between: each replay gives the bits of the eager calls."""
    graphs, states = [], []
    for k in range(2):
        s = _state(B, k)
        _calls(B, s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _calls(B, s)
        graphs.append(graph)
        states.append(s)
    for turn in range(4):
        for graph, s in zip(graphs, states):
            fresh = _state(B, 100 + 10 * turn)
            for k in INPUTS:
                s[k].copy_(fresh[k])
            for k in OUTPUTS:
                s[k].zero_()
            graph.replay()
            _calls(B, fresh)
            torch.cuda.synchronize()
            for k in OUTPUTS:
                assert torch.equal(s[k], fresh[k]), (turn, k)


def test_other_streams(B):
    """Two streams at once, given as an argument and as the current stream."""
    want = [_state(B, k) for k in range(2)]
    for s in want:
        _calls(B, s)
    torch.cuda.synchronize()
    states, streams = [_state(B, k) for k in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, stream in zip(states, streams):
            with torch.cuda.stream(stream):
                _calls(B, s)
    torch.cuda.synchronize()
    for s, w in zip(states, want):
        for k in OUTPUTS:
            assert torch.equal(s[k], w[k]), k
    s = states[0]
    s["y"].zero_()
    torch.cuda.synchronize()
    B.tabx_layer_norm(s["x"], s["w"], s["b"], EPS, s["y"], s["mean"], s["rstd"], s["on"], streams[1])
    streams[1].synchronize()
    assert torch.equal(s["y"], want[0]["y"])


def test_parts_draw_what_the_whole_batch_draws(B):
    env = _env(B, "c2_4096env_5v5", 64)
    E, N = env.E, env.N
    logits, u = torch.randn(E, N, 8, device=DEV), torch.rand(E, N, device=DEV)
    whole, halves = (torch.zeros(E, N, dtype=torch.uint8, device=DEV) for _ in range(2))
    how = B.TabxSampling(1.0, 0, 0.9)
    env.sample_actions(logits, how, u, whole)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for q, st in zip(env.parts(2), streams):
        sl = slice(q.first_env, q.first_env + q.E)
        q.sample_actions(logits[sl], how, u[sl], halves[sl], stream=st)
    torch.cuda.synchronize()
    assert torch.equal(whole, halves)
