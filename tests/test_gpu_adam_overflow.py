"""AdamW over many tensors with float states where v' or its mean is no finite float: the quotient is 0, as in the flat step's division."""
import math

import pytest
import torch

from ops_util import BF16, F32, close
from paper_2405_03637_b200 import binding as B
from test_gpu_adam_multi import GROUP, HYPER, Tensor, hyper

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rest", [B.REST_NONE, B.REST_BF16, B.REST_F32])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("inside", [False, True])
def test_an_infinite_v_moves_nothing_but_the_decay(rest, shift, inside):
    """x' = x - lr wd x, within a float's roundings of the decay (2^-23 of it) and of the stored form (a pair: 2^-8 of the second part; a master
    weight: 2^-24; a parameter alone: 2^-8)."""
    n = 3 * GROUP + 5
    t = Tensor(n, B.STATE_F32, rest, shift)
    at = torch.arange(0, n, 7, device="cuda")
    t.grad.t[at] = torch.where(torch.arange(len(at), device="cuda") % 2 == 0, 1e20, -3e30).to(BF16)
    x = (t.theta.t.double() + t.rest.t.double()) if rest == B.REST_BF16 else (t.rest.t if rest else t.theta.t).double()
    m64 = HYPER["beta1"] * t.m.t.double() + (1 - HYPER["beta1"]) * t.grad.t.double()
    plan = B.adam_plan_create([t.row()])
    B.adam_step(plan, hyper(B.FLAG_EPS_INSIDE_SQRT if inside else 0), 3)
    B.adam_plan_destroy(plan)
    assert (t.v.t[at] == math.inf).all() and int((t.v.t == math.inf).sum()) == len(at)
    close(t.m.t[at], m64[at], 2.0 ** -22 * m64[at].abs(), "m")
    decay = HYPER["lr"] * HYPER["weight_decay"] * x
    want, off = x - decay, 2.0 ** -22 * decay.abs()
    if rest == B.REST_BF16:
        hi, lo = t.theta.t.double(), t.rest.t.double()
        close((hi + lo)[at], want[at], (off + 2.0 ** -8 * 1.001 * (want - hi).abs())[at], "pair")
    elif rest == B.REST_F32:
        close(t.rest.t[at], want[at], (off + 2.0 ** -24 * 1.001 * want.abs())[at], "master")
    else:
        close(t.theta.t[at], want[at], (off + 2.0 ** -8 * 1.001 * want.abs())[at], "theta")
    for g in (t.theta, t.rest, t.m):
        assert g is None or g.t.float().isfinite().all()


@pytest.mark.parametrize("state,rest", [(B.STATE_F32, r) for r in (B.REST_NONE, B.REST_BF16, B.REST_F32)])
@pytest.mark.parametrize("shift", [0, 1])
def test_a_mean_of_v_that_overflows_under_the_root(state, rest, shift):
    """v' is a finite float, v' / (1 - beta2^t) is not: the root is infinite and the quotient 0; without weight decay nothing moves."""
    t = Tensor(2 * GROUP + 3, state, rest, shift)
    t.v.t.fill_(3e38)
    before = [None if g is None else g.t.clone() for g in (t.theta, t.rest)]
    plan = B.adam_plan_create([t.row()])
    B.adam_step(plan, hyper(B.FLAG_EPS_INSIDE_SQRT, weight_decay=0.0), 1)
    B.adam_plan_destroy(plan)
    assert t.v.t.isfinite().all()
    for g, b in zip((t.theta, t.rest), before):
        assert g is None or torch.equal(g.t, b)


@pytest.mark.parametrize("shift", [0, 1])
def test_what_is_no_number_stays_none(shift):
    """An infinite gradient makes inf / inf, a NaN a NaN; elements beside them are none the worse."""
    n = 2 * GROUP + 3
    t = Tensor(n, B.STATE_F32, B.REST_BF16, shift)
    t.grad.t[3], t.grad.t[GROUP + 9], t.grad.t[n - 1] = math.inf, math.nan, -math.inf
    plan = B.adam_plan_create([t.row()])
    B.adam_step(plan, hyper(), 2)
    B.adam_plan_destroy(plan)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[[3, GROUP + 9, n - 1]] = True
    assert t.theta.t[bad].isnan().all() and t.theta.t[~bad].isfinite().all() and t.rest.t[~bad].isfinite().all()
