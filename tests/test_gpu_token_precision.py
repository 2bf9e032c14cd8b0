"""Errors of token log-probabilities over rows of every kind: they have to be of both signs."""
import math

import pytest
import torch

from ops_util import BF16, F32
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
INF = math.inf
ROWS, VOCAB = 512, 13304


def rows_of(kind, g):
    """[ROWS, VOCAB] logits in 64 bits that bfloat16 holds, a target each."""
    rand = lambda *s: torch.rand(s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    pick = torch.arange(ROWS, device="cuda")
    if kind == "uniform":                       # equal logits, another number of them in each row
        z = torch.where(torch.arange(VOCAB, device="cuda") < (2 + (VOCAB - 2) * rand(ROWS, 1)).floor(), 3.0 * (rand(ROWS, 1) - 0.5), -INF)
        y = torch.zeros(ROWS, dtype=torch.int64, device="cuda")
    elif kind == "tied":                        # two values, both many times
        z = torch.where(rand(ROWS, VOCAB) < 0.5, 0.0, -6.0 * rand(ROWS, 1))
        y = pick % VOCAB
    elif kind == "peaked":                      # one logit far above the others, which are equal and weigh as much together
        z = torch.zeros(ROWS, VOCAB, device="cuda", dtype=torch.float64) - math.log(VOCAB) - 2 * (rand(ROWS, 1) - 0.5)
        z[pick, (rand(ROWS) * VOCAB).long()] = 0.0
        y = pick
    elif kind == "few":                         # seven logits are allowed
        z = torch.full((ROWS, VOCAB), -INF, device="cuda", dtype=torch.float64)
        at = torch.rand((ROWS, VOCAB), generator=g, device="cuda").topk(7).indices
        z.scatter_(1, at, 3.0 * torch.randn((ROWS, 7), generator=g, device="cuda", dtype=torch.float64))
        y = at[:, 0].contiguous()
    else:
        z = float(kind) * torch.randn((ROWS, VOCAB), generator=g, device="cuda", dtype=torch.float64)
        y = (rand(ROWS) * VOCAB).long()
    return z.to(BF16), y


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [0.05, 0.7, 1.0, 5.0])
@pytest.mark.parametrize("kind", ["uniform", "tied", "peaked", "few", "0.01", "2", "12"])
def test_errors_of_logp_are_of_both_signs(kind, tau, dtype):
    """The mean over 512 rows is within half a unit of a float's last place at 1, 2^-24.  A hardware exponential is off by up to 2^-22, the same way
    for the same logit.  A row's threads take theirs at offsets of their own, relative to what the hardware gives for the offset itself, so that a
    row's error is the mean over 256 threads of the difference of two such errors: with a spread of 2^-22 / sqrt(3) each, sqrt(2) 2^-22 / sqrt(3) / 16 =
    1.2e-8 for each row, all rows alike at worst.  A row of few logits has few threads, of its own choice: 2e-7 / sqrt(512) in the mean.  The sum's roundings
    are independent from row to row: 2^-23 / sqrt(512).  Four spreads of the largest are 4.9e-8, below 2^-24.  (Spread 0.01 and temperature 5: all
    exponentials within a hundredth.)  No row may be further off than the difference of two exponentials' errors, 2^-21, two factors between maxima, 2^-23
    each, and 16 roundings of a sum on its way through a thread's logits by twos (2 + 2), its turns (2 to 4), its halves, the division by the offset's power,
    the warp (5) and the block (3): together 1.7e-6, below 2^-19."""
    g = torch.Generator(device="cuda").manual_seed(len(kind))
    z, y = rows_of(kind, g)
    z64 = z.double() / tau
    want = z64.gather(1, y[:, None])[:, 0] - torch.logsumexp(z64, 1)
    logp, rest = torch.empty(ROWS, device="cuda"), torch.empty(ROWS, device="cuda")
    B.token_logp(z.to(dtype), y, tau, logp, logp_rest=rest)
    off = logp.double() + rest.double() - want
    there = want > -1e4                                      # (temperature 0.05: targets of no probability to speak of)
    assert off[there].abs().max() < 2.0 ** -19
    assert off[there].mean().abs() < 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_row_of_one_peak_is_exact(dtype):
    """Where all others have no weight, the peak's log-probability is 0 wherever it is in the row, and equal peaks share alike."""
    z = torch.full((300, 4001), -200.0, device="cuda", dtype=dtype)
    at = torch.arange(300, device="cuda") * 13
    z[torch.arange(300, device="cuda"), at] = 7.5
    logp, rest = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    B.token_logp(z, at, 1.0, logp, logp_rest=rest)
    assert (logp == 0).all() and (rest == 0).all()
    for k in (1, 2, 3, 5, 100):                              # k + 1 peaks: -log(k + 1), within a float's roundings of the sum
        z[:, 4001 - k:] = 7.5
        B.token_logp(z, at, 1.0, logp, logp_rest=rest)
        live = at < 4001 - k
        assert ((logp.double() + rest.double() + math.log(k + 1)).abs()[live] < 2.0 ** -23).all()
