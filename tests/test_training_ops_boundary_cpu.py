"""Refusals of the training-step operators, all detected on the host before any CUDA call (no GPU needed)."""
import ctypes

import pytest

from paper_2405_03637_b200 import binding as B

A = 0x100000                                    # never dereferenced: every call below fails validation first
SLOT = 0x100000                                 # arrays placed this far apart do not overlap


def at(i):
    return A + i * SLOT


def mat(i, rows, cols, ld=None, offset=0):
    return B.Matrix(at(i) + offset, rows, cols, cols if ld is None else ld)


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_struct_layouts():
    assert ctypes.sizeof(B.Matrix) == 32
    assert ctypes.sizeof(B.Distill) == 3 * 32 + 8 + 8


def test_norm_refusals(L):
    def call(x=mat(0, 4, 64), res=mat(1, 4, 64), w=at(2), eps=1e-5, ro=mat(3, 4, 64), y=mat(4, 4, 64), y8=None, s8=None, rstd=at(6)):
        return L.collage_add_rms_norm(x, res, w, eps, ro, y, y8, s8, rstd, None)
    assert call(x=None) == B.ERR_NULL
    assert call(w=None) == B.ERR_NULL
    assert call(y=None) == B.ERR_NULL                                     # no output at all
    assert call(y8=mat(5, 4, 64)) == B.ERR_NULL                           # 8 bits without a scale
    assert call(s8=at(5)) == B.ERR_ARG                                    # a scale without 8 bits
    assert call(res=None) == B.ERR_ARG                                    # residual_out without a residual
    for eps in (-1e-5, float("nan"), float("inf")):
        assert call(eps=eps) == B.ERR_ARG
    assert call(y=mat(4, 4, 63)) == B.ERR_ARG
    assert call(res=mat(1, 3, 64)) == B.ERR_ARG
    assert call(x=mat(0, 4, 64, ld=63)) == B.ERR_ARG
    assert call(x=mat(0, 4, 64, offset=1)) == B.ERR_ARG                   # half an element
    assert call(w=at(2) + 1) == B.ERR_ARG
    assert call(rstd=at(6) + 2) == B.ERR_ARG
    assert call(x=B.Matrix(None, 4, 64, 64)) == B.ERR_NULL
    assert call(x=mat(0, 1 << 31, 64), res=mat(1, 1 << 31, 64), ro=mat(3, 1 << 31, 64), y=mat(4, 1 << 31, 64)) == B.ERR_LIMIT
    assert call(x=mat(0, 4, 64, ld=1 << 41)) == B.ERR_LIMIT
    assert call(y=mat(1, 4, 64)) == B.ERR_ALIAS                           # y over the residual
    assert call(ro=mat(0, 4, 64, offset=2)) == B.ERR_ALIAS                # residual_out over part of x
    assert call(ro=mat(0, 4, 64, ld=65)) == B.ERR_ALIAS                   # x's array with another stride
    assert call(rstd=at(0) + 64) == B.ERR_ALIAS
    assert call(y=mat(3, 4, 64)) == B.ERR_ALIAS                           # two outputs in one place
    assert call(w=at(4) + 16) == B.ERR_ALIAS


def test_norm_backward_refusals(L):
    need = B.rms_norm_workspace_bytes(64)
    assert need > 0

    def call(dy=mat(0, 4, 64), r=mat(1, 4, 64), rstd=at(2), w=at(3), dres=mat(4, 4, 64), dx=mat(5, 4, 64), dw=at(6), ws=at(7), nb=need):
        return L.collage_add_rms_norm_backward(dy, r, rstd, w, dres, dx, dw, ws, nb, None)
    for k in ("dy", "r", "rstd", "w"):
        assert call(**{k: None}) == B.ERR_NULL
    assert call(dx=None, dw=None) == B.ERR_NULL
    assert call(ws=None) == B.ERR_WORKSPACE and call(nb=need - 1) == B.ERR_WORKSPACE and call(ws=at(7) + 8) == B.ERR_WORKSPACE
    assert call(r=mat(1, 4, 60)) == B.ERR_ARG
    assert call(dx=mat(5, 3, 64)) == B.ERR_ARG
    assert call(dx=mat(1, 4, 64)) == B.ERR_ALIAS                          # over r
    assert call(dx=mat(0, 4, 64, offset=16)) == B.ERR_ALIAS               # over part of dy
    assert call(dw=at(3)) == B.ERR_ALIAS
    assert call(ws=at(5)) == B.ERR_ALIAS


def test_quantize_refusals(L):
    x, q = mat(0, 4, 64), mat(1, 4, 64)
    assert L.collage_quantize_rows(None, q, at(2), None) == B.ERR_NULL
    assert L.collage_quantize_rows(x, q, None, None) == B.ERR_NULL
    assert L.collage_quantize_rows(x, mat(1, 4, 65), at(2), None) == B.ERR_ARG
    assert L.collage_quantize_rows(x, q, at(2) + 1, None) == B.ERR_ARG
    assert L.collage_quantize_rows(x, mat(0, 4, 64), at(2), None) == B.ERR_ALIAS


def test_gated_refusals(L):
    def call(x=mat(0, 5, 64), wg=mat(1, 24, 64), wu=mat(2, 24, 64), h=mat(3, 5, 24), gate=None, up=None, act=0):
        return L.collage_gated_ffn(x, wg, wu, h, gate, up, act, None)
    for k in ("x", "wg", "wu", "h"):
        assert call(**{k: None}) == B.ERR_NULL
    assert call(gate=mat(4, 5, 24)) == B.ERR_NULL                         # both or neither
    assert call(act=2) == B.ERR_ARG and call(act=-1) == B.ERR_ARG
    assert call(wu=mat(2, 23, 64)) == B.ERR_ARG
    assert call(x=mat(0, 5, 63)) == B.ERR_ARG
    assert call(h=mat(3, 5, 25)) == B.ERR_ARG
    assert call(gate=mat(4, 5, 24), up=mat(5, 5, 23)) == B.ERR_ARG
    assert call(h=mat(0, 5, 24)) == B.ERR_ALIAS
    assert call(gate=mat(4, 5, 24), up=mat(4, 5, 24)) == B.ERR_ALIAS
    # halves of one buffer: disjoint columns of one stride pass this check, overlapping ones do not
    assert call(gate=mat(4, 5, 24, ld=48), up=mat(4, 5, 24, ld=48, offset=46)) == B.ERR_ALIAS
    # 8 bits
    def call8(x=mat(0, 5, 64), sx=at(6), wg=mat(1, 24, 64), sg=at(7), wu=mat(2, 24, 64), su=at(8), h=mat(3, 5, 24), act=0):
        return L.collage_gated_ffn_e4m3(x, sx, wg, sg, wu, su, h, act, None)
    for k in ("x", "sx", "wg", "sg", "wu", "su", "h"):
        assert call8(**{k: None}) == B.ERR_NULL
    assert call8(act=7) == B.ERR_ARG and call8(sx=at(6) + 2) == B.ERR_ARG and call8(wg=mat(1, 24, 63)) == B.ERR_ARG
    assert call8(h=mat(1, 5, 24)) == B.ERR_ALIAS and call8(sx=at(3)) == B.ERR_ALIAS


def test_gated_backward_refusals(L):
    names = ("dh", "x", "wg", "wu", "gate", "up", "dg", "du", "dx", "dwg", "dwu")
    shapes = ((5, 24), (5, 64), (24, 64), (24, 64), (5, 24), (5, 24), (5, 24), (5, 24), (5, 64), (24, 64), (24, 64))

    def call(act=0, **kw):
        args = [kw.get(n, mat(i, *shapes[i])) for i, n in enumerate(names)]
        return L.collage_gated_ffn_backward(*args, act, None)
    for n in ("dh", "gate", "up", "dg", "du", "x", "wg", "wu", "dwg", "dwu"):
        assert call(**{n: None}) == B.ERR_NULL, n
    assert call(act=5) == B.ERR_ARG
    for n, i in (("gate", 4), ("dg", 6), ("dx", 8), ("dwg", 9), ("wu", 3)):
        assert call(**{n: mat(i, shapes[i][0], shapes[i][1] + 1)}) == B.ERR_ARG, n
    assert call(dg=mat(5, 5, 24)) == B.ERR_ALIAS                          # dgate in up's place
    assert call(dx=mat(1, 5, 64)) == B.ERR_ALIAS
    assert call(dwg=mat(2, 24, 64)) == B.ERR_ALIAS


def test_distill_refusals(L):
    def args(z=mat(0, 6, 100), i=mat(1, 6, 8), t=mat(2, 6, 8), dtype=B.DTYPE_BF16, index=4, temp=1.0):
        return ctypes.byref(B.Distill(z, i, t, dtype, index, temp))
    dz = mat(3, 6, 100)
    both = lambda a, d=dz, w=at(4), loss=at(5): L.collage_distill_loss_and_grad(a, w, loss, d, None)  # noqa: E731
    assert both(None) == B.ERR_NULL and both(args(), None) == B.ERR_NULL and both(args(), w=None) == B.ERR_NULL and both(args(), loss=None) == B.ERR_NULL
    assert both(args(dtype=2)) == B.ERR_ARG and both(args(index=2)) == B.ERR_ARG
    for temp in (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e60):
        assert both(args(temp=temp)) == B.ERR_ARG
    assert both(args(t=mat(2, 6, 7))) == B.ERR_ARG and both(args(i=mat(1, 5, 8), t=mat(2, 5, 8))) == B.ERR_ARG
    assert both(args(), mat(3, 6, 99)) == B.ERR_ARG
    assert both(args(i=mat(1, 6, 1025), t=mat(2, 6, 1025))) == B.ERR_LIMIT
    assert both(args(), mat(0, 6, 100, offset=2)) == B.ERR_ALIAS          # shifted over the logits
    assert both(args(), mat(1, 6, 100)) == B.ERR_ALIAS                    # over the indexes
    assert both(args(), loss=at(4)) == B.ERR_ALIAS                        # the loss over the weights
    assert both(args(), w=at(4) + 2) == B.ERR_ARG
    assert L.collage_distill_loss(args(), None, None, None) == B.ERR_NULL
    assert L.collage_distill_loss(args(), at(5), at(5), None) == B.ERR_ALIAS
    assert L.collage_distill_loss_backward(args(), None, at(4), dz, None) == B.ERR_NULL
    assert L.collage_distill_loss_backward(args(), at(5), None, dz, None) == B.ERR_NULL
    assert L.collage_distill_loss_backward(args(dtype=B.DTYPE_F32), at(5), at(4), mat(3, 6, 100, offset=2), None) == B.ERR_ARG
