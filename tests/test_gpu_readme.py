"""The learner's example of README.md, run as it stands there: its gradients against 64-bit formulas, with
all memory that nobody has written yet full of NaN (needs an MI355X)."""
import os
import re

import pytest
import torch

from paper_2602_01665_amd import inputs as I
from tests import learner_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _block(of):
    with open(README) as f:
        found = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if of in b]
    assert len(found) == 1
    return found[0]


@pytest.fixture
def untouched_memory_is_nan():
    torch.use_deterministic_algorithms(True, warn_only=True)       # and with it, empty() fills
    assert bool(torch.empty(3, device=DEV).isnan().all())
    yield
    torch.use_deterministic_algorithms(False)


@pytest.mark.filterwarnings("ignore")
def test_the_update_has_the_gradients_of_its_rows(untouched_memory_is_nan):
    from paper_2602_01665_amd.binding import TabxEnv
    w = I.WORKLOADS["c2_4096env_5v5"]
    env = TabxEnv(I.make_params(w, 60, max_steps=20), I.make_scenario(w, 60))
    env.reset()
    env.observe()
    E, N, D = env.E, env.N, env.D
    scripted = env.sc["team"].view(E, N)
    policy = I.policy("medium", seed=1)
    env.prime_scripted(policy, scripted)
    g = torch.Generator(device=DEV).manual_seed(2)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    m = (n(D, 9) / D ** 0.5).requires_grad_()
    weight, bias, adv = 1 + 0.1 * n(D), 0.1 * n(D), n(E, N)
    names = dict(torch=torch, env=env, scripted=scripted, policy=policy, weight=weight, bias=bias,
                 actions=torch.zeros(E, N, dtype=torch.uint8, device=DEV), network=lambda rows: rows.float() @ m,
                 loss_gradients=lambda lp, old, h: (-adv * torch.exp(lp - old), torch.full_like(h, -0.01)))
    before = env.obs.clone(), env.amask.clone()
    exec(compile(_block("env.norm_obs"), README, "exec"), names)

    on = names["ours"].cpu().view(-1).double()
    y = names["y"].detach().cpu().double().view(E * N, D)
    taken, mask = names["taken"].cpu().view(-1).long(), before[1].cpu().view(-1)
    gl, ge = -adv.cpu().double().view(-1) * on, torch.full((E * N,), -0.01, dtype=torch.float64) * on
    assert torch.equal(names["old_log_prob"][names["ours"] != 0], names["log_prob"][names["ours"] != 0])   # the first ratio is one
    q, rows = m.detach().cpu().double().requires_grad_(), y.clone().requires_grad_()
    l = torch.where((mask == 0)[:, None] & (torch.arange(8) == R.ATTACK), -1e300, (rows @ q)[:, :8] / float(0.9))
    lp = torch.log_softmax(l, 1)
    ent = -torch.where(lp > -1e200, lp.exp() * lp, 0.0).sum(1)
    (gl * lp.gather(1, taken[:, None])[:, 0] + ge * ent).sum().backward()
    # logits in 32 bits are off by a sum of D products, the shares by as much and the steps of an exponential (64 of
    # them), and the shares' gradients by that times eight logarithms; the product over rows adds E N terms
    size = (y.abs() @ q.detach().abs()).amax(1) + 8
    off = ((D + 64) * R.U * size * (gl.abs() + 8 * ge.abs()) * 8 / 0.9)[:, None]
    bound = (y.abs() * off).sum(0)[:, None] + (E * N + 8) * R.U * (y.abs() * (gl.abs() + 8 * ge.abs())[:, None]).sum(0)[:, None] / 0.9
    got = m.grad.cpu().double()
    assert bool(((got - q.grad).abs()[:, :8] <= bound).all()) and bool((got[:, 8] == 0).all())
    # the rows' gradient comes in bf16, off by 2^-8 of itself; then sums over rows
    dy = rows.grad * on[:, None]
    x = before[0].cpu().double().view(E * N, D)
    c = x - x.mean(1, keepdim=True)
    h = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5)
    d_dy = (2.0 ** -8 + 2.0 ** -20) * dy.abs() + 9 * off * q.detach().abs().amax(1)[None] * on[:, None]
    for name, want, part in (("grad_weight", (dy * h).sum(0), h.abs()), ("grad_bias", dy.sum(0), torch.ones_like(h))):
        bound = (d_dy * part).sum(0) + (E * N + 64) * R.U * (dy.abs() * (part + 4)).sum(0)
        assert bool(((names[name].cpu().double() - want).abs() <= bound).all()), name
    assert not torch.equal(env.obs, before[0])                     # the tick has been on since


def test_the_curriculum_draws_from_its_scores():
    from paper_2602_01665_amd import binding as B
    names = dict(torch=torch, B=B, I=I, TabxEnv=B.TabxEnv, w=I.WORKLOADS["c2_4096env_5v5"])
    exec(compile(_block("sample_levels"), README, "exec"), names)
    bank = names["bank"]
    bank.dones.fill_(1)
    bank.sample_levels(names["scores"], B.TabxSampling(0.3, top_k=100), torch.rand(bank.E, device=DEV), env_mask=bank.dones)
    assert int(bank.st["next_level"].max()) < 100                  # equal scores: the first hundred
