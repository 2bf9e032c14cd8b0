"""Refusals of the block norm's backward pass from x, all detected on the host before any CUDA call."""
import pytest
import torch

from paper_2405_03637_b200 import binding as B
from test_alignment_ops_binding_cpu import COL, MAT, ROW, calls, refused  # noqa: F401
from test_alignment_ops_boundary_cpu import at, mat, norm_in
from test_training_ops_binding_cpu import Fake, FakeStream, elsewhere


def test_refusals():
    L, need = B.lib(), B.block_norm_workspace_bytes(64)

    def call(s=norm_in(), dy=mat(4, 4, 64), dr=mat(5, 4, 64), x=mat(6, 4, 64), rpost=at(7), rpre=at(8), dx=mat(9, 4, 64), do=mat(10, 4, 64),
             dg=mat(11, 1, 64), dpost=at(12), dpre=at(13), ws=at(14), nb=need):
        return L.collage_block_norm_backward_from_x(s, dy, dr, x, rpost, rpre, dx, do, dg, dpost, dpre, ws, nb, None)
    assert call(s=None) == B.ERR_NULL and call(dy=None, dr=None, dpre=None) == B.ERR_NULL
    assert call(x=None) == B.ERR_NULL and call(rpre=None) == B.ERR_NULL and call(rpost=None) == B.ERR_NULL and call(s=norm_in(pre=None)) == B.ERR_NULL
    assert call(dy=None) == B.ERR_ARG                                     # dpre_weight without a gradient of y
    assert call(x=mat(6, 4, 63)) == B.ERR_ARG and call(x=mat(6, 4, 64, offset=1)) == B.ERR_ARG
    assert call(ws=None) == B.ERR_WORKSPACE and call(nb=need - 1) == B.ERR_WORKSPACE
    assert call(dx=mat(6, 4, 64)) == B.ERR_ALIAS                          # over x
    assert call(do=mat(9, 4, 64)) == B.ERR_ALIAS and call(ws=at(6)) == B.ERR_ALIAS and call(dpost=at(6)) == B.ERR_ALIAS


def test_the_binding_takes_x_in_the_place_of_r(calls):  # noqa: F811
    f = lambda r, **kw: B.block_norm_backward(MAT, r, MAT, ROW, ROW, MAT, MAT, post_weight=COL, pre_weight=COL, **kw)  # noqa: E731
    f(None, x=MAT)
    f(MAT)
    assert calls.count == 2
    for bad in (elsewhere(MAT, 1), elsewhere(MAT, -1), Fake(4, 64, dtype=torch.float16)):
        refused(f, None, x=bad)
    refused(f, MAT, x=MAT)                                                # one or the other
    refused(f, None, x=MAT, stream=FakeStream(0x5000, device=1))
    assert calls.count == 2
