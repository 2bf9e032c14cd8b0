"""Exponents of the gradients of the token losses."""
import math

import pytest
import torch

from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu


def worst_temperature():
    """A temperature around 1 at which log2(e) / t is just below a float, so that the next one down lacks nearly a whole unit of its last place."""
    return max((k / 4096 for k in range(4096, 6144)), key=lacking)


def lacking(t):
    c = 1.4426950408889634 / t
    near = float(torch.tensor(c, dtype=torch.float64).float())
    unit = 2.0 ** (math.floor(math.log2(c)) - 23)
    return (1 - (near - c) / unit) if near >= c else -1.0


def test_exponents_of_the_gradient():
    """q_j of logits 8 to 14 below the maximum, multiples of 1 / 64, so that the difference is exact.  log2(e) / t to the nearest float is half a unit of its
    last place off at most, here less than a twentieth; rounded down it would lack all of a unit, 2^-23 / c of x = 11 log2(e) / t, which makes q 1e-6 too
    large on average.  The product's rounding is of both signs, an exponential 2^-22 off at most: the mean error is below 3e-7."""
    t = worst_temperature()
    assert lacking(t) > 0.95
    rows, vocab = 64, 4096
    g = torch.Generator(device="cuda").manual_seed(4)
    z = -8.0 - torch.randint(0, 384, (rows, vocab), generator=g, device="cuda") / 64
    z[:, 0] = 0
    y = torch.full((rows,), 1, device="cuda")
    one, d, back = torch.ones(rows, device="cuda"), torch.empty_like(z), torch.empty_like(z)
    loss, logp, stats = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    want = -torch.softmax(z.double() / t, 1) / t
    B.policy_loss_and_grad(z, y, t, -one, one, loss, d)                  # coefficient 1
    B.token_logp(z, y, t, logp, stats=stats)
    B.token_logp_backward(z, y, t, stats, one, back)
    for got in (d, back):
        assert (got.double()[:, 2:] / want[:, 2:] - 1).mean().abs() < 3e-7
