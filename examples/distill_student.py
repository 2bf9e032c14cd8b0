"""Trains a small student on a teacher's top logits with the training-step operators and Collage AdamW.

    python examples/distill_student.py [--steps 60] [--tokens 512] [--width 256] [--ffn 640] [--layers 2] [--vocab 4099]

The student is an embedding, blocks of (residual + RMS norm, gated feed-forward, down projection), a last norm and an output
projection.  Everything between the matrix products of torch runs in this package: `add_rms_norm`, `gated_ffn`,
`distill_loss_and_grad` and their backward passes write bfloat16 gradients, which the multi-tensor Collage-plus step
consumes.  Afterwards the same weights are evaluated in 8 bits (`quantize_rows`, the norm's 8-bit output, `gated_ffn_e4m3`).

The teacher is a fixed random table: for each token its logits over the vocabulary, of which the student sees the top ones.
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
from paper_2405_03637_b200 import binding as B  # noqa: E402

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS, TEMPERATURE = 1e-5, 2.0


class Student:
    """Parameters, their gradients and optimizer state, and the activations of one batch, all allocated once."""

    def __init__(self, tokens, width, ffn, layers, vocab, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std: (torch.randn(s, generator=g, device="cuda") * std).to(BF16)  # noqa: E731
        self.tokens, self.width, self.ffn, self.layers, self.vocab = tokens, width, ffn, layers, vocab
        self.p = {"embed": rand(vocab, width, std=1.0), "norm": torch.ones(width, dtype=BF16, device="cuda"),
                  "head": rand(vocab, width, std=0.02)}
        for i in range(layers):
            self.p[f"{i}.norm"] = torch.ones(width, dtype=BF16, device="cuda")
            self.p[f"{i}.gate"], self.p[f"{i}.up"] = rand(ffn, width, std=width ** -0.5), rand(ffn, width, std=width ** -0.5)
            self.p[f"{i}.down"] = rand(width, ffn, std=ffn ** -0.5)
        self.grad = {n: torch.zeros_like(t) for n, t in self.p.items()}
        state = {n: [torch.zeros_like(t) for _ in range(4)] for n, t in self.p.items()}      # delta-theta, m, v, delta-v
        self.state = state
        self.plan = B.plan_create([(t, state[n][0], state[n][1], state[n][2], state[n][3], self.grad[n], t.numel())
                                   for n, t in self.p.items()])
        new = lambda *s, dtype=BF16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
        self.blocks = [dict(r=new(tokens, width), y=new(tokens, width), rstd=new(tokens, dtype=F32), h=new(tokens, ffn),
                            gate=new(tokens, ffn), up=new(tokens, ffn)) for _ in range(layers)]
        self.last = dict(r=new(tokens, width), y=new(tokens, width), rstd=new(tokens, dtype=F32))
        self.logits, self.loss = new(tokens, vocab), new(tokens, dtype=F32)
        self.workspace = torch.empty(B.rms_norm_workspace_bytes(width), dtype=torch.uint8, device="cuda")

    def forward(self, ids):
        x, residual = torch.zeros(self.tokens, self.width, dtype=BF16, device="cuda"), self.p["embed"][ids]
        for i, b in enumerate(self.blocks):
            B.add_rms_norm(x, residual, self.p[f"{i}.norm"], EPS, residual_out=b["r"], y=b["y"], rstd=b["rstd"])
            B.gated_ffn(b["y"], self.p[f"{i}.gate"], self.p[f"{i}.up"], b["h"], gate=b["gate"], up=b["up"])
            x, residual = b["h"] @ self.p[f"{i}.down"].T, b["r"]
        B.add_rms_norm(x, residual, self.p["norm"], EPS, residual_out=self.last["r"], y=self.last["y"], rstd=self.last["rstd"])
        torch.matmul(self.last["y"], self.p["head"].T, out=self.logits)

    def backward(self, ids, top_index, top_logits, row_weight):
        dlogits = self.logits                    # the gradient takes the logits' place
        B.distill_loss_and_grad(self.logits, top_index, top_logits, TEMPERATURE, row_weight, self.loss, dlogits)
        torch.matmul(dlogits.T, self.last["y"], out=self.grad["head"])
        dy = dlogits @ self.p["head"]
        dr = torch.empty_like(dy)
        B.add_rms_norm_backward(dy, self.last["r"], self.last["rstd"], self.p["norm"], dr, self.grad["norm"], self.workspace)
        for i in reversed(range(self.layers)):
            b = self.blocks[i]
            torch.matmul(dr.T, b["h"], out=self.grad[f"{i}.down"])
            dh, dy = dr @ self.p[f"{i}.down"], torch.empty_like(dr)
            B.gated_ffn_backward(dh, b["y"], self.p[f"{i}.gate"], self.p[f"{i}.up"], b["gate"], b["up"], b["gate"], b["up"], dx=dy,
                                 dw_gate=self.grad[f"{i}.gate"], dw_up=self.grad[f"{i}.up"])
            B.add_rms_norm_backward(dy, b["r"], b["rstd"], self.p[f"{i}.norm"], dr, self.grad[f"{i}.norm"], self.workspace, dresidual=dr)
        self.grad["embed"].zero_().index_add_(0, ids, dr)

    def step(self, t, lr):
        B.adamw_step_multi(self.plan, B.make_hyper(lr, 0.9, 0.999, 1e-8, 0.01), t, B.PLUS)

    def logits_in_8_bits(self, ids):
        """The same network with 8-bit operands in its gated products."""
        x, residual = torch.zeros(self.tokens, self.width, dtype=BF16, device="cuda"), self.p["embed"][ids]
        y8 = torch.empty(self.tokens, self.width, dtype=E4M3, device="cuda")
        scale = torch.empty(self.tokens, dtype=F32, device="cuda")
        for i in range(self.layers):
            r, h = torch.empty_like(residual), torch.empty(self.tokens, self.ffn, dtype=BF16, device="cuda")
            w = []
            for name in ("gate", "up"):
                w8 = torch.empty(self.ffn, self.width, dtype=E4M3, device="cuda")
                ws = torch.empty(self.ffn, dtype=F32, device="cuda")
                B.quantize_rows(self.p[f"{i}.{name}"], w8, ws)
                w += [w8, ws]
            B.add_rms_norm(x, residual, self.p[f"{i}.norm"], EPS, residual_out=r, y8=y8, y8_scale=scale)
            B.gated_ffn_e4m3(y8, scale, *w, h)
            x, residual = h @ self.p[f"{i}.down"].T, r
        y = torch.empty_like(x)
        B.add_rms_norm(x, residual, self.p["norm"], EPS, y=y)
        return y @ self.p["head"].T


def run(steps=60, tokens=512, width=256, ffn=640, layers=2, vocab=4099, top=16, lr=3e-3, seed=0):
    """Mean loss per token after each step, and at the end in bfloat16 and in 8 bits."""
    student = Student(tokens, width, ffn, layers, vocab, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    known = 256                                                                   # distinct tokens in the data
    table = torch.randn(known, vocab, generator=g, device="cuda") * 3
    teacher_logits, teacher_index = table.topk(top, dim=1)
    losses = []
    for t in range(1, steps + 1):
        ids = torch.randint(0, known, (tokens,), generator=g, device="cuda")
        weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
        weight[::17] = 0                                                          # positions that do not count
        student.forward(ids)
        student.backward(ids, teacher_index[ids], teacher_logits[ids].contiguous(), weight)
        student.step(t, lr)
        losses.append(student.loss.sum())                                         # (read at the end: no wait in the loop)
    ids = torch.arange(tokens, device="cuda") % known
    at, tl = teacher_index[ids], teacher_logits[ids].contiguous()
    student.forward(ids)
    loss, loss8 = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    B.distill_loss(student.logits, at, tl, TEMPERATURE, loss)
    B.distill_loss(student.logits_in_8_bits(ids), at, tl, TEMPERATURE, loss8)
    B.plan_destroy(student.plan)
    if code := B.pipeline_fault():                                                # (waits for the GPU: at the end, or at a checkpoint)
        raise RuntimeError(f"a kernel gave up a wait (code {code}): weights and losses are undefined")
    return [x.item() for x in losses], loss.mean().item(), loss8.mean().item()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 60), ("tokens", 512), ("width", 256), ("ffn", 640), ("layers", 2), ("vocab", 4099)):
        ap.add_argument(f"--{name}", type=int, default=default)
    curve, loss, loss8 = run(**vars(ap.parse_args()))
    for t in range(0, len(curve), max(1, len(curve) // 10)):
        print(f"step {t + 1:4d}  loss {curve[t]:.4f}")
    print(f"after training: {loss:.4f} in bfloat16, {loss8:.4f} with 8-bit gated products")
