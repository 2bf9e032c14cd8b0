"""Kernels of alignment training that walk over their work: many turns, several groups of threads in a block, each form of the outputs.

The definitions and tolerances are those of the tests of the single operators.
"""
import math

import pytest
import torch

from ops_util import BF16, E4M3, U, close, normal
from paper_2405_03637_b200 import binding as B
from test_gpu_block_norm import EPS, FORMS, Case, check_backward, check_forward, vec
from test_gpu_token_losses import Rows
from test_gpu_token_losses import test_logp_and_its_backward_match_definition as logp_matches
from test_gpu_token_losses import test_policy_matches_definition as policy_matches

pytestmark = pytest.mark.gpu

# rows for four turns and more of 148 blocks, with ten groups of 96 threads in each, eight of 128, four of 256, three of 320 and two of 512
WALKS = [(6001, 1032), (5300, 1544), (2400, 4096), (1800, 5120), (1300, 8192)]
NO_TOKEN_GATE = [f for f in FORMS if f[0] != "token"]


@pytest.mark.parametrize("rows,cols", WALKS)
@pytest.mark.parametrize("form", NO_TOKEN_GATE, ids=str)
def test_block_norm_walks(rows, cols, form):
    """y and its 8 bits, both norms, either one alone (which has a barrier of its own), and none."""
    check_forward(Case(rows, cols, 0, 0, form), out8=True)
    check_forward(Case(rows, cols, 8, 0, form, seed=7), out8=False)


@pytest.mark.parametrize("place", ["x", "block", "y"])
@pytest.mark.parametrize("rows,cols", [(6001, 1032), (2400, 4096)])
def test_block_norm_walks_in_place(rows, cols, place):
    for form in NO_TOKEN_GATE[:2]:
        check_forward(Case(rows, cols, 0, 0, form), in_place=place)


@pytest.mark.parametrize("rows,cols", [(6001, 1032), (2400, 4096)])
def test_block_norm_walks_over_rows_whose_squares_no_float_holds(rows, cols):
    """Among ordinary rows, in every group: their sums are taken again, times a power of two."""
    size = torch.ones(rows, 1, device="cuda")
    for k, v in enumerate((1e25, 3e38, 1e-25, 1e-37)):
        size[k::9] = v
    o = (normal(1, rows, cols, dtype=torch.float32).clamp(-1, 1) * size).to(BF16)
    x, one = torch.zeros_like(o), torch.ones(cols, dtype=BF16, device="cuda")
    r, y, y8, scale = torch.empty_like(o), torch.empty_like(o), torch.empty_like(o, dtype=E4M3), vec(rows)
    want = o.double() / torch.sqrt((o.double() ** 2).mean(1, keepdim=True))
    B.block_norm(x, o, r, post_weight=one, pre_weight=one, y=y, eps=0.0)
    close(r, want, U * 1.01 * want.abs(), "r")
    B.block_norm(o, x, r, pre_weight=one, y=y, y8=y8, y8_scale=scale, eps=0.0)
    close(y, want, U * 1.01 * want.abs(), "y")
    close(scale, want.abs().amax(1) / 448, 2.0 ** -18 * want.abs().amax(1) / 448, "scale")
    close(y8.double() * scale.double()[:, None], want, want.abs() * (2.0 ** -4 + 2.0 ** -17) + scale.double()[:, None] * 2.0 ** -10 * 1.001, "y8")
    assert torch.equal(r, o)


@pytest.mark.parametrize("rows,cols", [(1300, 257), (1300, 1001), (1200, 4095)])
def test_rows_that_are_not_whole_vectors_take_several_turns(rows, cols):
    """592 blocks forward, 296 backward."""
    for form in (FORMS[0], FORMS[1], FORMS[3], FORMS[5]):
        check_forward(Case(rows, cols, 0, 0, form), out8=True)
        check_backward(Case(rows, cols, 0, 0, form, seed=3), use_dy=form[3])


# more turns than stages, with 15 groups of a warp, 8 of 64 threads, 4 of 128, 2 of 256, and one row at a time of 640 and 768 threads
@pytest.mark.parametrize("rows,cols", [(13500, 136), (6500, 520), (3700, 2048), (2400, 4096), (900, 5120), (900, 5128), (900, 6144), (900, 8192)])
@pytest.mark.parametrize("form", [FORMS[0], FORMS[1], FORMS[2]], ids=str)
def test_block_norm_backward_refills_its_stages(rows, cols, form):
    check_backward(Case(rows, cols, 0, 0, form))


@pytest.mark.parametrize("rows,vocab", [(320, 12000), (302, 50257), (1001, 9001), (600, 32000)])
def test_token_losses_with_a_block_of_256_threads_for_each_row(rows, vocab):
    policy_matches(rows, vocab, 0, 0)
    logp_matches(rows, vocab, 0, 0)


def test_policy_of_many_rows_with_several_blocks_each():
    """Rows too long for L2 to keep those under way: 800 of 65536 floats, two blocks and more for each."""
    r = Rows(800, 65536, 0, 0, torch.float32, 1.0)
    adv, w = normal(1, 800, dtype=torch.float32), torch.rand(800, device="cuda")
    loss, logp, d = vec(800), vec(800), r.box()
    B.policy_loss_and_grad(r.z.t, r.y, 1.0, adv, w, loss, d.t, logp=logp)
    live = r.counts & (w != 0)
    close(logp, torch.where(live, r.logp, 0.0), r.logp_off, "logp")
    coef = torch.where(live, -adv.double() * w.double(), 0.0)
    want, tol = r.gradient(coef, 2.0 ** -22 * coef.abs())
    close(d.t, want, tol, "dlogits")
    close(loss, coef, 2.0 ** -22 * coef.abs(), "loss")
    assert d.untouched_outside() and math.isfinite(float(loss.sum()))
