"""AdamW over bfloat16 pairs: theta' is the bfloat16 nearest to theta + rest - lr (q + weight_decay (theta + rest)), and rest' what that lacks.

q is the float quotient that the documentation has, formed here by the same float operations one by one (torch rounds each); the sum is formed in 64
bits.  What a kernel may be off: the decay's two roundings and its product's, 2^-22 of the decay; q by a unit of its last place where the root is
not the nearest float (a few in a million), 2^-22 of lr q; the rounding of the sum's second float, 2^-46 of the sum.  Elements that lie nearer
to half-way than that are left out, a few in a million; a sum in one float, 2^-24 off, would put one in 2^17 on the wrong side.
"""
import math

import pytest
import torch

from ops_util import BF16, F32, close, normal
from paper_2405_03637_b200 import binding as B
from test_gpu_adam_multi import GROUP, Tensor, hyper, spacing

pytestmark = pytest.mark.gpu
LR = 1e-5


def f32(v):
    return float(torch.tensor(v, dtype=torch.float64).float())


def quotient(t, step, inside, eps, beta1=0.9, beta2=0.999):
    """Float operations, each rounded: m' / bc1 over sqrt(v' / bc2) + eps."""
    one = lambda v: torch.tensor(f32(v), device="cuda")  # noqa: E731
    g = t.grad.t.float()
    if t.state == B.STATE_F32:
        m, v = t.m.t.clone(), t.v.t.clone()
    else:
        each = lambda s: s.t.repeat_interleave(GROUP)[:t.n]  # noqa: E731
        m, v = t.m.t.float() * each(t.m_scale), t.v.t.float() * each(t.v_scale)
        v = v * v
    m = m * one(beta1) + g * one(1 - beta1)
    v = v * one(beta2) + (g * g) * one(1 - beta2)
    bc1, bc2 = 1 - beta1 ** step, 1 - beta2 ** step
    num = m * one(1 / bc1)
    den = (v.double() * f32(1 / bc2) + f32(eps)).float().sqrt() if inside else v.sqrt() * one(1 / math.sqrt(bc2)) + one(eps)
    return num / den


def nearest(x):
    """Nearest bfloat16 values, ties to even, in 64 bits."""
    s = spacing(x, 8)
    return torch.round(x / s) * s


@pytest.mark.parametrize("state", [B.STATE_E4M3, B.STATE_F32])
@pytest.mark.parametrize("n,shift", [(1 << 22, 0), ((1 << 21) + 3, 1)])
@pytest.mark.parametrize("inside,decay", [(False, 0.1), (False, 0.0), (True, 0.0)])
def test_theta_is_the_nearest_value_and_rest_what_it_lacks(state, n, shift, inside, decay):
    step, eps = 7, 1e-8 if not inside else 1e-12
    t = Tensor(n, state, B.REST_BF16, shift, seed=31)
    q = quotient(t, step, inside, eps).double()
    pair = t.theta.t.double() + t.rest.t.double()
    x = pair - LR * q - LR * decay * pair
    once = (t.theta.t.float() + (t.rest.t.float() - f32(LR) * q.float())).to(BF16).double()
    plan = B.adam_plan_create([t.row()])
    B.adam_step(plan, hyper(B.FLAG_EPS_INSIDE_SQRT if inside else 0, lr=LR, weight_decay=decay, eps=eps), step, seed=3)
    B.adam_plan_destroy(plan)
    off = 2.0 ** -22 * (LR * decay * pair.abs() + LR * q.abs()) + 2.0 ** -46 * x.abs()
    near = nearest(x)
    open_ = ((x - near).abs() - spacing(x, 8) / 2).abs() < off
    assert open_.float().mean() < 1e-5
    theta, rest = t.theta.t.double(), t.rest.t.double()
    assert ((theta == near) | open_).all()
    assert ((theta - x).abs() <= spacing(x, 8) / 2 + off).all()
    close(rest, x - theta, 2.0 ** -8 * 1.001 * (x - theta).abs() + 1.01 * off, "rest")
    if decay == 0.0:
        assert int(((once != near) & ~open_).sum()) > 0                 # one float for the sum would not do on these values
    assert t.intact()


@pytest.mark.parametrize("state", [B.STATE_E4M3, B.STATE_F32])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("lr", [2.0 ** -50, 2.0 ** -34, 0.0])
def test_sums_half_way_go_by_the_update(state, shift, lr):
    """theta + rest exactly half-way between two bfloat16 values, and an update far below a float's last place, of either sign: the nearest value is
    the one on the update's side; without an update the even one.  theta + rest is exact in a float, and so is what the update adds to it in a second one: no
    element is left out."""
    n = 8 * GROUP + 77                              # whole groups and one that is cut short
    t = Tensor(n, state, B.REST_BF16, shift)
    g = torch.Generator(device="cuda").manual_seed(5)
    mantissa, power = torch.randint(1, 128, (n,), generator=g, device="cuda"), torch.randint(-3, 1, (n,), generator=g, device="cuda")
    sign = lambda: torch.randint(0, 2, (n,), generator=g, device="cuda") * 2.0 - 1.0  # noqa: E731
    value = sign() * (128 + mantissa) * torch.exp2(power - 7.0)
    half = sign() * torch.exp2(power - 8.0)
    t.theta.t.copy_(value), t.rest.t.copy_(half), t.grad.t.copy_(sign())
    assert torch.equal(t.theta.t.double(), value.double()) and torch.equal(t.rest.t.double(), half.double())
    for s in (t.m, t.v, t.m_scale, t.v_scale):
        if s is not None:
            s.t.zero_()
    q = quotient(t, 1, False, 1e-8).double()
    x = value.double() + half.double() - lr * q
    assert lr == 0 or (x != value.double() + half.double()).all()
    plan = B.adam_plan_create([t.row()])
    B.adam_step(plan, hyper(lr=lr, weight_decay=0.0), 1)
    B.adam_plan_destroy(plan)
    assert torch.equal(t.theta.t.double(), nearest(x))
    close(t.rest.t, x - nearest(x), 2.0 ** -8 * 1.001 * half.double().abs(), "rest")
    assert t.intact()
