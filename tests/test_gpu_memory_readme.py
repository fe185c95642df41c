"""The memory's example of README.md, run as it stands there: the ticks at once against its steps, its gradients against
64-bit formulas, with all memory that nobody has written yet full of NaN (needs an MI355X)."""
import os
import re

import pytest
import torch

from paper_2602_01665_amd import inputs as I
from tests import memory_reference as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


@pytest.fixture
def untouched_memory_is_nan():
    torch.use_deterministic_algorithms(True, warn_only=True)       # and with it, empty() fills
    assert bool(torch.empty(3, device=DEV).isnan().all())
    yield
    torch.use_deterministic_algorithms(False)


@pytest.mark.filterwarnings("ignore")
def test_the_memory_and_its_gradients(untouched_memory_is_nan):
    from paper_2602_01665_amd.binding import TabxEnv
    with open(README) as f:
        found = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "env.remember" in b]
    assert len(found) == 1
    w = I.WORKLOADS["c2_4096env_5v5"]
    env = TabxEnv(I.make_params(w, 20, max_steps=5), I.make_scenario(w, 20))
    env.reset()
    env.observe()
    env.dones.zero_()
    W, H, K, V = 48, 4, 32, 32
    g = torch.Generator(device=DEV).manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    inward, product, steps = n(env.D, W) / env.D ** 0.5 / 10, n(W, H * (2 * K + V)) / W ** 0.5, []

    def project(y):
        both, v = (y.float() @ product).bfloat16().split((2 * H * K, H * V), -1)
        return both.unflatten(-1, (2 * H, K)), v.unflatten(-1, (H, V))

    def choose(stream, out):
        steps.append(out.clone())
        return torch.randint(0, 8, (env.E, env.N), generator=g, device=DEV).to(torch.uint8)

    names = dict(torch=torch, env=env, W=W, gain=1 + 0.1 * n(W), project=project, choose=choose,
                 embed=lambda obs: ((obs @ inward).bfloat16(), n(env.E, env.N, W).bfloat16()),
                 loss_gradients=lambda stream, outs: (n(*outs.shape).bfloat16(), n(*stream.shape).bfloat16()))
    exec(compile(found[0], README, "exec"), names)

    T, E, N = names["T"], env.E, env.N
    rows = lambda t: t.detach().cpu().reshape(T, E * N, *t.shape[3:])  # noqa: E731
    q, k, v, go = rows(names["q"]), rows(names["k"]), rows(names["vs"]), rows(names["grad_outs"])
    fresh = names["fresh"].cpu()
    assert bool((fresh != 0).any())
    args = (names["log_decay"].cpu(), names["scale"], fresh, names["before"].cpu().view(E * N, H, K, V))
    want = M.attention(q, k, v, *args)
    M.near(rows(names["outs"]), *want["out"], "all ticks at once")
    M.near(rows(torch.stack(steps)), *want["out"], "step by step")
    M.near(names["state"].cpu().view(E * N, H, K, V), *want["state_out"], "state")
    back = M.attention_grad(q, k, v, *args, go, None)
    for name, got in (("grad_q", names["grad_qk"][..., :H, :]), ("grad_k", names["grad_qk"][..., H:, :]), ("grad_v", names["grad_vs"])):
        M.near(rows(got), *back[name], name)
