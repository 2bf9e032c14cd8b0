"""Aligns a small policy with rewards and with preferences, on the operators of alignment training.

    python examples/align_policy.py [--steps 60] [--tokens 512] [--width 256] [--ffn 640] [--layers 2] [--vocab 4099]

The policy is an embedding, blocks of (gated feed-forward, down projection) with a norm before and after each, a learned gate for each
channel and scaled residuals, and an output projection.  Between the matrix products of torch everything runs in this package:
`block_norm`, `gated_ffn` and their backward passes; first the clipped policy loss on tokens that the policy itself samples
(`policy_loss_and_grad`), then the preference loss of pairs of answers (`token_logp`, `preference_loss`, `token_logp_backward`).  The gradients, clipped
to a norm, go into AdamW with 8-bit states over bfloat16 pairs (`adam_grad_norm`, `adam_step`).

A token is answered well if it is the one that a fixed random table has for the token before it.
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
from paper_2405_03637_b200 import binding as B  # noqa: E402

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS, BLOCK_SCALE = 1e-5, 0.5


class Policy:
    """Parameters, their gradients and optimizer state, and the activations of one batch, all allocated once."""

    def __init__(self, tokens, width, ffn, layers, vocab, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std: (torch.randn(s, generator=g, device="cuda") * std).to(BF16)  # noqa: E731
        ones = lambda *s: torch.ones(s, dtype=BF16, device="cuda")  # noqa: E731
        self.tokens, self.layers = tokens, layers
        self.p = {"embed": rand(vocab, width, std=1.0), "norm": ones(width), "head": rand(vocab, width, std=width ** -0.5)}
        for i in range(layers):
            self.p[f"{i}.gate"], self.p[f"{i}.up"] = rand(ffn, width, std=width ** -0.5), rand(ffn, width, std=width ** -0.5)
            self.p[f"{i}.down"] = rand(width, ffn, std=ffn ** -0.5)
            self.p[f"{i}.post"], self.p[f"{i}.pre"], self.p[f"{i}.channel"] = ones(width), ones(width), ones(1, width)
        self.grad = {n: torch.zeros_like(t) for n, t in self.p.items()}
        zeros = lambda n, dtype: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
        groups = lambda t: -(-t.numel() // B.ADAM_GROUP)  # noqa: E731
        self.state = [(t, torch.zeros_like(t), zeros(t.numel(), E4M3), zeros(t.numel(), E4M3), zeros(groups(t), F32), zeros(groups(t), F32), self.grad[n])
                      for n, t in self.p.items()]
        self.plan = B.adam_plan_create(self.state)
        new = lambda *s, dtype=BF16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
        self.first = dict(y=new(tokens, width), rstd=new(tokens, dtype=F32))
        self.blocks = [dict(h=new(tokens, ffn), gate=new(tokens, ffn), up=new(tokens, ffn), o=new(tokens, width), r=new(tokens, width), y=new(tokens, width),
                            rstd_post=new(tokens, dtype=F32), rstd_pre=new(tokens, dtype=F32)) for _ in range(layers)]
        self.logits, self.loss, self.logp = new(tokens, vocab), new(tokens, dtype=F32), new(tokens, dtype=F32)
        self.norm, self.grad_scale = new(1, dtype=F32), new(1, dtype=F32)
        self.workspace = torch.empty(max(B.block_norm_workspace_bytes(width), B.rms_norm_workspace_bytes(width)), dtype=torch.uint8, device="cuda")
        self.sums = torch.empty(B.workspace_bytes(), dtype=torch.uint8, device="cuda")
        B.workspace_init(self.sums)

    def norms(self, i):
        return dict(gate=self.p[f"{i}.channel"], post_weight=self.p[f"{i}.post"], pre_weight=self.p[f"{i}.pre"], block_scale=BLOCK_SCALE)

    def forward(self, ids):
        self.r0 = self.p["embed"][ids]
        B.add_rms_norm(self.r0, None, self.p["norm"], EPS, y=self.first["y"], rstd=self.first["rstd"])
        r, y = self.r0, self.first["y"]
        for i, b in enumerate(self.blocks):
            B.gated_ffn(y, self.p[f"{i}.gate"], self.p[f"{i}.up"], b["h"], gate=b["gate"], up=b["up"])
            torch.matmul(b["h"], self.p[f"{i}.down"].T, out=b["o"])
            B.block_norm(r, b["o"], b["r"], y=b["y"], rstd_post=b["rstd_post"], rstd_pre=b["rstd_pre"], eps=EPS, **self.norms(i))
            r, y = b["r"], b["y"]
        torch.matmul(y, self.p["head"].T, out=self.logits)

    def backward(self, ids, dlogits):
        """Gradients of all parameters from that of the logits."""
        y = self.blocks[-1]["y"] if self.blocks else self.first["y"]
        torch.matmul(dlogits.T, y, out=self.grad["head"])
        dy, dr = dlogits @ self.p["head"], None
        for i in reversed(range(self.layers)):
            b, before, x = self.blocks[i], (self.blocks[i - 1]["y"] if i else self.first["y"]), (self.blocks[i - 1]["r"] if i else self.r0)
            dx, do = torch.empty_like(dy), torch.empty_like(dy)
            g = {n: self.grad[f"{i}.{k}"] for n, k in (("dgate", "channel"), ("dpost_weight", "post"), ("dpre_weight", "pre"))}
            B.block_norm_backward(dy, None, b["o"], b["rstd_post"], b["rstd_pre"], dx, do, dr=dr, workspace=self.workspace, x=x, **g, **self.norms(i))
            dr = dx
            torch.matmul(do.T, b["h"], out=self.grad[f"{i}.down"])
            dh, dy = do @ self.p[f"{i}.down"], torch.empty_like(dx)
            B.gated_ffn_backward(dh, before, self.p[f"{i}.gate"], self.p[f"{i}.up"], b["gate"], b["up"], b["gate"], b["up"], dx=dy,
                                 dw_gate=self.grad[f"{i}.gate"], dw_up=self.grad[f"{i}.up"])
        dembed = torch.empty_like(dy)
        B.add_rms_norm_backward(dy, self.r0, self.first["rstd"], self.p["norm"], dembed, self.grad["norm"], self.workspace, dresidual=dr)
        self.grad["embed"].zero_().index_add_(0, ids, dembed)

    def policy_step(self, ids, target, advantage, row_weight, old_logp=None, ref_logp=None):
        """Loss of sampled tokens and its gradients; the gradient of the logits takes their place."""
        self.forward(ids)
        B.policy_loss_and_grad(self.logits, target, 1.0, advantage, row_weight, self.loss, self.logits, old_logp=old_logp, ref_logp=ref_logp,
                               kl_weight=0.0 if ref_logp is None else 0.02, logp=self.logp)
        self.backward(ids, self.logits)

    def log_probabilities(self, ids, target):
        self.forward(ids)
        B.token_logp(self.logits, target, 1.0, self.logp)
        return self.logp.clone()

    def preference_step(self, ids, target, offsets, ref_logp, beta):
        """Losses of pairs of answers, each over their number, and their gradients."""
        self.forward(ids)
        new = lambda *s: torch.empty(s, dtype=F32, device="cuda")  # noqa: E731
        stats, rest, grad, loss = new(self.tokens, 2), new(self.tokens), new(self.tokens), new(offsets.numel() // 2)
        B.token_logp(self.logits, target, 1.0, self.logp, stats=stats, logp_rest=rest)
        B.preference_loss(self.logp, target, self.logits.shape[1], offsets, beta, loss, grad_logp=grad, ref_logp=ref_logp, logp_rest=rest,
                          pair_weight=torch.full_like(loss, 1.0 / loss.numel()))
        B.token_logp_backward(self.logits, target, 1.0, stats, grad, self.logits)
        self.backward(ids, self.logits)
        return loss

    def step(self, t, lr, max_norm=1.0):
        B.adam_grad_norm(self.plan, max_norm, self.norm, self.grad_scale, self.sums)
        B.adam_step(self.plan, B.make_hyper(lr, 0.9, 0.99, 1e-8, 0.01), t, seed=1, grad_scale=self.grad_scale)


def run(steps=60, tokens=512, width=256, ffn=640, layers=2, vocab=4099, lr=2e-3, pairs=8, seed=0):
    """Share of good answers among the sampled tokens before each step on rewards, and the pairs' mean loss before each of half as many on preferences."""
    policy = Policy(tokens, width, ffn, layers, vocab, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    known = min(64, vocab)                                                          # tokens that occur
    answer = torch.randint(0, known, (known,), generator=g, device="cuda")
    draw = lambda: torch.randint(0, known, (tokens,), generator=g, device="cuda")  # noqa: E731
    rewards, losses = [], []
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    for t in range(1, steps + 1):
        ids = draw()
        policy.forward(ids)
        # half of the tokens are the policy's own, the others explore
        sampled = torch.multinomial(policy.logits.float().softmax(1), 1, generator=g)[:, 0]
        target = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.5, sampled, draw())
        reward = (target == answer[ids]).float()
        target[::17] = -1                                                            # positions that do not count
        old = policy.log_probabilities(ids, target)
        policy.policy_step(ids, target, reward - reward.mean(), weight, old_logp=old, ref_logp=old)
        policy.step(t, lr)
        rewards.append((sampled == answer[ids]).float().mean())
    ids = draw()
    good, bad = answer[ids], draw()
    offsets = torch.arange(2 * pairs + 1, device="cuda") * (tokens // (2 * pairs))
    which = torch.arange(tokens, device="cuda") // (tokens // (2 * pairs)) % 2
    target = torch.where(which == 0, good, bad)
    ref = policy.log_probabilities(ids, target)
    for t in range(steps + 1, steps + 1 + steps // 2):
        losses.append(policy.preference_step(ids, target, offsets, ref, 0.1).sum())
        policy.step(t, lr)
    B.adam_plan_destroy(policy.plan)
    if code := B.pipeline_fault():                                                  # (waits for the GPU: at the end, or at a checkpoint)
        raise RuntimeError(f"a kernel gave up a wait (code {code}): weights and losses are undefined")
    return [x.item() for x in rewards], [x.item() for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 60), ("tokens", 512), ("width", 256), ("ffn", 640), ("layers", 2), ("vocab", 4099)):
        ap.add_argument(f"--{name}", type=int, default=default)
    rewards, losses = run(**vars(ap.parse_args()))
    for t in range(0, len(rewards), max(1, len(rewards) // 10)):
        print(f"step {t + 1:4d}  share of good answers {rewards[t]:.4f}")
    for t in range(0, len(losses), max(1, len(losses) // 5)):
        print(f"pairs {t + 1:4d}  loss {losses[t]:.4f}")
