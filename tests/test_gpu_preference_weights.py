"""Pairs that are masked by a weight of 0 take no part, whatever their log-probabilities are."""
import math

import pytest
import torch

from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.mark.parametrize("smooth", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("average", [False, True])
def test_a_pair_of_weight_zero_takes_no_part(smooth, average):
    logp = torch.tensor([-INF, 0.0, -INF, -INF, NAN, -1.0, 0.0, -INF, -2.0, -3.0], device="cuda")
    y, o = torch.zeros(10, dtype=torch.int64, device="cuda"), torch.arange(11, device="cuda")
    w = torch.tensor([0.0, 0.0, -0.0, 0.0, 1.0], device="cuda")
    loss, ratio, grad = (torch.full((k,), NAN, device="cuda") for k in (5, 5, 10))
    B.preference_loss(logp, y, 9, o, 0.5, loss, grad_logp=grad, pair_weight=w, label_smoothing=smooth, average=average, log_ratio=ratio)
    assert (loss[:4] == 0).all() and (grad[:8] == 0).all()
    assert ratio[0] == -INF and ratio[1].isnan() and ratio[2].isnan() and ratio[3] == INF and ratio[4] == 1
    alone, own = torch.full((1,), NAN, device="cuda"), torch.full((2,), NAN, device="cuda")
    B.preference_loss(logp[8:].clone(), y[8:].clone(), 9, o[:3].clone(), 0.5, alone, grad_logp=own, label_smoothing=smooth, average=average)
    assert torch.equal(loss[4:], alone) and torch.equal(grad[8:], own)


def test_and_its_rows_get_no_gradient_of_the_logits():
    """A token of probability 0 in a pair that is masked: zeros all the way."""
    z = torch.randn(4, 300, device="cuda")
    z[0, 5] = z[1, 5] = -INF
    y, o = torch.full((4,), 5, device="cuda"), torch.arange(5, device="cuda")
    w = torch.tensor([0.0, 1.0], device="cuda")
    logp, stats, loss, grad, d = (torch.empty(*s, device="cuda") for s in ((4,), (4, 2), (2,), (4,), (4, 300)))
    B.token_logp(z, y, 1.0, logp, stats=stats)
    B.preference_loss(logp, y, 300, o, 0.1, loss, grad_logp=grad, pair_weight=w)
    B.token_logp_backward(z, y, 1.0, stats, grad, d)
    assert loss[0] == 0 and (d[:2] == 0).all() and d.isfinite().all() and (d[2:] != 0).any()
