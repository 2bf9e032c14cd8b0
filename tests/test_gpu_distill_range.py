"""Distillation of rows whose values lie far from zero: what counts is how logits differ within a row.

The definition in 64 bits is taken on logits (and teacher's logits) less their row's largest, which changes neither
probabilities nor loss and is exact for these inputs; lse gets the largest back.  The tolerances know the differences only.
"""
import math

import pytest
import torch

from ops_util import BF16, F32, U, close, distill64, normal
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
NAN = math.nan


def teacher(seed, rows, vocab, k):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(rows, vocab, generator=g, device="cuda").topk(k, dim=1).indices, torch.randn(rows, k, generator=g, device="cuda") * 3


def check(z, at, top, tau, what):
    rows, vocab = z.shape
    zmax = z.double().amax(1, keepdim=True)
    d, e = z.double() - zmax, top.double() - top.double().amax(1, keepdim=True)
    loss64, lse64, grad64 = distill64(d, at, e, tau)
    lse64 = lse64 + zmax[:, 0] / tau
    # The argument of a student's exponential is a difference times 1 / (tau ln 2) less a logarithm below 2^5: five roundings of
    # 2^-24 each relative to the difference, two relative to the logarithm; the sums (vocab / 64 + 16) 2^-23; twice all that.
    rel = 2.0 ** -19 + (vocab / 64 + 16) * 2.0 ** -22
    a, q = (-d / tau).clamp_max(90), torch.softmax(d / tau, 1)
    p = torch.softmax(e / tau, 1)
    # p = exp(-b) / sum is off by p (b 2^-22 + 2^-21), where p b <= 0.37; twice that
    entries = torch.zeros_like(q).scatter_(1, at, p * 2.0 ** -20 + 0.37 * 2.0 ** -21)
    weight = torch.linspace(0.25, 1.25, rows, device="cuda")
    want = grad64 * weight.double()[:, None]
    tol = tau * weight.double()[:, None] * (q * (a * 2.0 ** -21 + rel) + entries + 2.0 ** -100)
    if z.dtype == BF16:
        tol = tol + U * 1.001 * want.abs()
    terms = (p * (2 * -d.gather(1, at) / tau - 2 * e / tau + 20)).nan_to_num(0).sum(1)
    ltol = tau * tau * (2.0 ** -21 * terms + 2 * rel)
    loss, lse, dz = (torch.full(s, NAN, device="cuda") for s in ((rows,), (rows,), (1,)))
    dz = torch.full_like(z, NAN)
    B.distill_loss(z, at, top, tau, loss, lse=lse)
    close(loss, loss64, ltol, what + " loss")
    close(lse, lse64, 2 * rel + 2.0 ** -22 * lse64.abs(), what + " lse")
    B.distill_loss_backward(z, at, top, tau, lse, weight, dz)
    close(dz, want, tol, what + " gradient in a call of its own")
    loss, dz = torch.full_like(loss, NAN), torch.full_like(z, NAN)
    B.distill_loss_and_grad(z, at, top, tau, weight, loss, dz)
    close(dz, want, tol, what + " gradient in one pass")
    close(loss, loss64 * weight.double(), ltol * weight.double(), what + " loss in one pass")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,k", [(4, 1031, 9), (300, 1031, 9), (5, 33_001, 20), (2, 900_001, 5)])
def test_rows_of_logits_far_from_zero(rows, vocab, k, dtype):
    spread = normal(rows + vocab, rows, vocab, std=2.0, dtype=F32)
    at, top = teacher(1, rows, vocab, k)
    for tau in (0.05, 0.7, 4.0) if vocab < 100_000 else (0.7,):
        for far in (-1e9, -1e5, -1e3, 1e3, 1e5, 1e6, 1e12, 1e20):
            z = (spread + far).to(dtype)                     # (from 1e5 on, where a unit of the type is larger than that, mostly all alike)
            z[1::2, ::7] -= abs(far) * 2.0 ** -7             # and in every other row a seventh of them a unit of bfloat16 below
            check(z, at, top, tau, f"{far:g} at {tau}:")


@pytest.mark.parametrize("rows,vocab,k", [(3, 1031, 9), (3, 90_001, 40)])
def test_teachers_logits_far_from_zero(rows, vocab, k):
    z = normal(3, rows, vocab, std=2.0)
    at, spread = teacher(2, rows, vocab, k)
    lowest = torch.finfo(F32).min
    for tau in (0.5, 0.7, 3.0):
        for far in (-1e9, -1e6, 1e4, 1e6, 1e20):
            check(z, at, spread + far, tau, f"{far:g} at {tau}:")
        top = spread.clone()
        top[0] = lowest                                      # all alike: a uniform teacher
        top[1, 1:] = lowest                                  # one entry has all the mass
        check(z, at, top, tau, f"lowest at {tau}:")
