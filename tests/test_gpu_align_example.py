"""The alignment example: that it runs, and its gradients against autograd in 64 bits."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("align_policy", Path(__file__).resolve().parent.parent / "examples" / "align_policy.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs(example):
    rewards, losses = example.run(steps=6, tokens=96, width=64, ffn=128, layers=2, vocab=301, pairs=3)
    assert len(rewards) == 6 and len(losses) == 3 and all(math.isfinite(x) for x in rewards + losses)


def logits64(example, p, ids, layers):
    norm = lambda t: t / torch.sqrt((t * t).mean(1, keepdim=True) + example.EPS)  # noqa: E731
    r = p["embed"][ids]
    y = norm(r) * p["norm"]
    for i in range(layers):
        gate = y @ p[f"{i}.gate"].T
        o = (gate * torch.sigmoid(gate) * (y @ p[f"{i}.up"].T)) @ p[f"{i}.down"].T
        r = r + example.BLOCK_SCALE * p[f"{i}.channel"] * norm(o) * p[f"{i}.post"]
        y = norm(r) * p[f"{i}.pre"]
    return y @ p["head"].T


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_gradients_of_the_whole_against_autograd(example, kind):
    """Two layers of bfloat16 activations (each rounded to 2^-9 on average) put the gradients about 1 % from the exact ones; 5 % in the 2-norm
    leaves room for that and for nothing that is wrong."""
    tokens, layers, vocab = 64, 2, 257
    policy = example.Policy(tokens, 64, 96, layers, vocab, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    for n, t in policy.p.items():                      # weights and gates that are not all ones
        if n.split(".")[-1] in ("norm", "post", "pre", "channel"):
            t.mul_(1 + 0.3 * torch.randn(t.shape, generator=g, device="cuda"))
    ids, target = (torch.randint(0, vocab, (tokens,), generator=g, device="cuda") for _ in range(2))
    target[::9] = -1
    counts, at = target >= 0, target.clamp_min(0)
    p = {n: t.double().requires_grad_() for n, t in policy.p.items()}
    logp = logits64(example, p, ids, layers).log_softmax(1).gather(1, at[:, None])[:, 0]
    logp = torch.where(counts, logp, 0.0)
    if kind == "policy":
        advantage = torch.randn(tokens, generator=g, device="cuda")
        weight = torch.rand(tokens, generator=g, device="cuda") / tokens
        policy.policy_step(ids, target, advantage, weight)
        (-(logp - logp.detach()).exp() * advantage * weight * counts).sum().backward()
    else:
        offsets = torch.tensor([0, 20, 40, 50, 64], device="cuda")
        ref = (logp.detach() + torch.randn(tokens, generator=g, device="cuda") * counts).float()
        policy.preference_step(ids, target, offsets, ref, 0.3)
        s = [(logp - ref.double())[a:b].sum() for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())]
        (-sum(torch.nn.functional.logsigmoid(0.3 * (s[2 * i] - s[2 * i + 1])) for i in range(2)) / 2).backward()
    for n, t in policy.grad.items():
        want = p[n].grad
        assert float((t.double() - want).norm()) <= 0.05 * float(want.norm()), n
    example.B.adam_plan_destroy(policy.plan)
