"""Helpers of the tests of the training-step operators: strided matrices inside guarded buffers, 64-bit definitions."""
from __future__ import annotations

import math

import torch

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
U = 2.0 ** -8                 # largest relative error of one rounding to bfloat16 (8 significant bits)


class Box:
    """A [rows, cols] view with row stride `ld`, `shift` elements into a buffer filled with a sentinel byte."""

    def __init__(self, rows, cols, dtype=BF16, ld=None, shift=0, data=None):
        self.rows, self.cols, self.ld = rows, cols, ld or cols
        size = torch.empty(0, dtype=dtype).element_size()
        self.lo, self.size = 256 // size + shift, size
        total = self.lo + max(rows, 1) * self.ld + 256 // size
        self.raw = torch.full((total * size,), 0x5B, dtype=torch.uint8, device="cuda")
        flat = self.raw.view(dtype)
        self.t = flat[self.lo:self.lo + max(rows, 1) * self.ld].as_strided((rows, cols), (self.ld, 1))
        if data is not None:
            self.t.copy_(data)

    def untouched_outside(self) -> bool:
        """Nothing but the matrix's own elements was written."""
        inside = torch.zeros(self.raw.numel() // self.size, dtype=torch.bool, device="cuda")
        if self.rows and self.cols:
            inside[self.lo:self.lo + self.rows * self.ld].as_strided((self.rows, self.cols), (self.ld, 1)).fill_(True)
        keep = ~inside.repeat_interleave(self.size)
        return bool((self.raw[keep] == 0x5B).all())


def normal(seed, *shape, std=1.0, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def close(got, want, tol, what=""):
    """|got - want| <= tol elementwise, all in 64 bits; non-finite values have to agree."""
    got, want = got.double(), want.double()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(want)
    both_nan = got.isnan() & want.isnan()
    bad = ~(((got - want).abs() <= tol) | (got == want) | both_nan)
    if bad.any():
        i = bad.flatten().nonzero()[0].item()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: got {got.flatten()[i].item()!r} "
                             f"want {want.flatten()[i].item()!r} tol {tol.flatten()[i].item():.3g}")


def act_and_slope64(kind, g):
    """0 = SiLU, 1 = GELU by tanh; value and derivative in 64 bits."""
    if kind == 0:
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return g / 2 * (1 + t), (1 + t) / 2 + g / 2 * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def distill64(z, index, top, tau):
    """Per-row loss, log-sum-exp, and d loss / d logits of the definition, row by row in 64 bits."""
    z = z.double().cpu() / tau
    index, top = index.cpu().long(), top.double().cpu() / tau
    rows, vocab = z.shape
    loss, lse, grad = torch.zeros(rows, dtype=torch.float64), torch.logsumexp(z, 1), torch.zeros_like(z)
    for i in range(rows):
        there = (index[i] >= 0) & (index[i] < vocab)
        at, t = index[i][there], top[i][there]
        if t.numel() == 0 or bool((t == -math.inf).all()):
            continue
        logp = t - torch.logsumexp(t, 0)
        p = logp.exp()
        terms = p * (logp - (z[i, at] - lse[i]))
        loss[i] = tau * tau * terms[p != 0].sum()
        grad[i] = tau * (z[i] - lse[i]).exp()
        grad[i].index_add_(0, at, -tau * p)
    return loss.cuda(), lse.cuda(), grad.cuda()
