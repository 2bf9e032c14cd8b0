"""Training-step operators on the GPU against their definitions in 64 bits.

Tolerances.  One rounding to bfloat16 is at most 2^-8 of the value.  A float sum of K terms is at most K 2^-23 of the sum of
their magnitudes off (twice the usual bound, for sums that truncate).  Each is stated where it is used.
"""
import math

import pytest
import torch

from ops_util import BF16, E4M3, F32, U, Box, act_and_slope64, close, distill64, normal
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5
INF, NAN = math.inf, math.nan


def vec(n, dtype=F32):
    return torch.full((n,), NAN, dtype=F32, device="cuda").to(dtype)


# ------------------------------------------------------------------------------------------------- residual + RMS norm ---

ROW_SHAPES = [(1, 1), (3, 7), (2, 8), (5, 64), (4, 100), (33, 257), (7, 768), (3, 1000), (130, 1024), (1, 4096), (19, 4096), (9, 5120),
              (3, 8192), (2, 11008), (5, 16384), (2, 20008), (2, 40003)]
# (row stride beyond the columns, elements off a 16-byte boundary)
LAYOUTS = [(0, 0), (8, 0), (3, 0), (0, 1)]


def check_norm(rows, cols, pad, shift, residual, seed=0, out8=True, in_place=False):
    box = lambda dtype=BF16, data=None: Box(rows, cols, dtype, cols + pad, shift, data)  # noqa: E731
    x, res = box(data=normal(seed, rows, cols, std=3.0)), box(data=normal(seed + 1, rows, cols)) if residual else None
    weight = normal(seed + 2, cols)
    ro, y, y8 = box() if residual else None, box(), box(E4M3) if out8 else None
    scale, rstd = vec(rows), vec(rows)
    r64 = x.t.double() + (res.t.double() if residual else 0)
    if in_place:
        ro, y = (res if residual else None), x
    B.add_rms_norm(x.t, res.t if residual else None, weight, EPS, residual_out=ro.t if residual else None, y=y.t,
                   y8=y8.t if out8 else None, y8_scale=scale if out8 else None, rstd=rstd)
    rstd64 = 1 / torch.sqrt((r64 * r64).mean(1) + EPS)
    y64 = r64 * rstd64[:, None] * weight.double()
    # r: two bfloat16 values added in float (2^-24), one rounding.  rstd: the sum of squares is K/256 + 10 roundings deep per
    # thread at most, so its half power is well inside K 2^-24; y: that, two products, one rounding
    if residual:
        close(ro.t, r64, U * r64.abs() * 1.001, "residual_out")
    deep = (cols / 32 + 16) * 2.0 ** -23
    close(rstd, rstd64, deep * rstd64, "rstd")
    close(y.t, y64, (U * 1.001 + deep) * y64.abs(), "y")
    if out8:
        scale64 = y64.abs().amax(1) / 448
        close(scale, scale64, (deep + 2.0 ** -22) * scale64, "scale")
        # 4 significant bits: half a unit is 2^-4 of the value, and 2^-10 of the scale among the subnormals
        close(y8.t.double() * scale.double()[:, None], y64, y64.abs() * (2.0 ** -4 + 4 * deep) + scale64[:, None] * 2.0 ** -10 * 1.001, "y8")
        assert y8.untouched_outside()
    for b in (x, res, ro, y):
        assert b is None or b.untouched_outside()


@pytest.mark.parametrize("rows,cols", ROW_SHAPES)
@pytest.mark.parametrize("pad,shift", LAYOUTS)
def test_norm_matches_definition(rows, cols, pad, shift):
    check_norm(rows, cols, pad, shift, residual=True)
    check_norm(rows, cols, pad, shift, residual=False, seed=9, out8=False)


@pytest.mark.parametrize("rows,cols", [(300, 64), (1025, 136), (301, 520), (700, 1024), (310, 257), (400, 4096), (299, 8192), (330, 16384), (300, 20000)])
def test_norm_and_quantise_many_rows(rows, cols):
    check_norm(rows, cols, 0, 0, residual=True)
    check_norm(rows, cols, 8, 0, residual=False, seed=3)
    x, q, scale = Box(rows, cols, BF16, cols, 0, normal(5, rows, cols, std=0.02)), Box(rows, cols, E4M3), vec(rows)
    B.quantize_rows(x.t, q.t, scale)
    amax = x.t.float().abs().amax(1)
    assert torch.equal(scale, amax / torch.full_like(amax, 448))
    assert torch.equal(q.t.view(torch.uint8), (x.t.float() / scale[:, None]).to(E4M3).view(torch.uint8)) and q.untouched_outside()


@pytest.mark.parametrize("rows,cols", [(5, 64), (3, 1000), (3, 4096), (2, 5121), (2, 40000)])
def test_norm_in_place(rows, cols):
    check_norm(rows, cols, 0, 0, residual=True, in_place=True)
    check_norm(rows, cols, 0, 0, residual=False, in_place=True)


def test_norm_rows_of_zeros_and_non_finite_values():
    x = normal(3, 6, 512)
    x[1] = 0
    x[2, 5] = INF
    x[3, 7] = NAN
    x[4] *= 1e-30
    weight = torch.ones(512, dtype=BF16, device="cuda")
    y, y8, scale = torch.empty_like(x), torch.empty_like(x, dtype=E4M3), vec(6)
    B.add_rms_norm(x, None, weight, EPS, y=y, y8=y8, y8_scale=scale)
    assert (y[1] == 0).all() and (y8[1].float() == 0).all() and scale[1] == 0
    assert y[3].isnan().all() and y8[3].float().isnan().all() and scale[3].isnan()
    assert y[2, 5].isnan() and scale[2].isnan()             # infinity times 1 / infinity
    for i in (0, 4, 5):
        want = x[i].double() / torch.sqrt((x[i].double() ** 2).mean() + EPS)
        close(y[i], want, U * 1.01 * want.abs(), f"row {i}")


@pytest.mark.parametrize("rows,cols", ROW_SHAPES + [(300, 64), (1025, 136), (700, 1024)])
@pytest.mark.parametrize("pad,shift", LAYOUTS)
def test_norm_backward_matches_definition(rows, cols, pad, shift):
    box = lambda data=None: Box(rows, cols, BF16, cols + pad, shift, data)  # noqa: E731
    dy, r, dres = box(normal(1, rows, cols)), box(normal(2, rows, cols, std=2.0)), box(normal(3, rows, cols))
    weight = normal(4, cols)
    rstd = (1 / torch.sqrt((r.t.double() ** 2).mean(1) + EPS)).float()
    ws = torch.full((B.rms_norm_workspace_bytes(cols),), 0xFF, dtype=torch.uint8, device="cuda")
    n = r.t.double() * rstd.double()[:, None]
    g = dy.t.double() * weight.double()
    c = (g * n).mean(1, keepdim=True)
    dw64, mag = (dy.t.double() * n).sum(0), (dy.t.double() * n).abs().sum(0)
    spread = (g * n).abs().mean(1, keepdim=True)             # the mean's own error is cols 2^-24 of this at most
    for use_res in (True, False):
        dx, dweight = box(), vec(cols, BF16)
        B.add_rms_norm_backward(dy.t, r.t, rstd, weight, dx.t, dweight, ws, dresidual=dres.t if use_res else None)
        want = rstd.double()[:, None] * (g - n * c) + (dres.t.double() if use_res else 0)
        terms = rstd.double()[:, None] * (g.abs() + (n * c).abs()) + (dres.t.double().abs() if use_res else 0)
        tol = U * 1.001 * want.abs() + 2.0 ** -20 * terms + rstd.double()[:, None] * n.abs() * spread * (cols / 32 + 16) * 2.0 ** -23
        close(dx.t, want, tol, "dx")
        close(dweight, dw64, U * 1.001 * dw64.abs() + (rows + 8) * 2.0 ** -23 * mag, "dweight")
        assert dx.untouched_outside()
        # one output at a time, and dx in the place of an input, give the same bits
        only = box()
        B.add_rms_norm_backward(dy.t, r.t, rstd, weight, only.t, None, None, dresidual=dres.t if use_res else None)
        assert torch.equal(only.t, dx.t)
        only_w = vec(cols, BF16)
        B.add_rms_norm_backward(dy.t, r.t, rstd, weight, None, only_w, ws)
        assert torch.equal(only_w, dweight)
        place = box(dres.t if use_res else dy.t)
        if use_res:
            B.add_rms_norm_backward(dy.t, r.t, rstd, weight, place.t, only_w, ws, dresidual=place.t)
        else:
            B.add_rms_norm_backward(place.t, r.t, rstd, weight, place.t, only_w, ws)
        assert torch.equal(place.t, dx.t) and torch.equal(only_w, dweight)


def test_norm_gradient_agrees_with_differences():
    rows, cols = 3, 24
    x, weight, dy = normal(1, rows, cols), normal(2, cols), normal(3, rows, cols)
    y, rstd, dx, dweight = torch.empty_like(x), vec(rows), torch.empty_like(x), vec(cols, BF16)
    B.add_rms_norm(x, None, weight, EPS, y=y, rstd=rstd)
    B.add_rms_norm_backward(dy, x, rstd, weight, dx, dweight, torch.empty(B.rms_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda"))

    def objective(x, w):
        return (dy.double() * x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * w).sum()
    step = 1e-5
    for t, grad in ((x, dx), (weight, dweight)):
        for i in range(t.numel()):
            a, b = (x.double(), weight.double())
            e = torch.zeros(t.numel(), dtype=torch.float64, device="cuda")
            e[i] = step
            e = e.view_as(t)
            d = (objective(a + e, b) - objective(a - e, b)) / (2 * step) if t is x else (objective(a, b + e) - objective(a, b - e)) / (2 * step)
            # one rounding, and the differences' own error (third derivative and cancellation), below 1e-4 here
            assert abs(grad.flatten()[i].item() - d.item()) <= U * abs(d.item()) + 1e-4


@pytest.mark.parametrize("rows,cols", ROW_SHAPES)
@pytest.mark.parametrize("pad,shift", LAYOUTS)
def test_quantize_rows(rows, cols, pad, shift):
    x = Box(rows, cols, BF16, cols + pad, shift, normal(5, rows, cols, std=0.02))
    x.t[rows // 2] = 0
    q, scale = Box(rows, cols, E4M3, cols + pad, shift), vec(rows)
    B.quantize_rows(x.t, q.t, scale)
    amax = x.t.float().abs().amax(1)
    assert torch.equal(scale, amax / torch.full_like(amax, 448))         # one float division (a Python scalar would be inverted first)
    want = torch.where(scale[:, None] > 0, x.t.float() / scale[:, None], 0.0).to(E4M3)
    assert torch.equal(q.t.view(torch.uint8), want.view(torch.uint8))
    assert q.untouched_outside()


def test_quantize_rows_every_value_of_the_format_and_non_finite_rows():
    x = torch.zeros(5, 300, dtype=BF16, device="cuda")
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(E4M3).float()
    codes = codes[~codes.isnan()]
    x[0, :codes.numel()] = codes.to(BF16)                    # with 448 as the largest the scale is 1: every code maps to itself
    x[1, 3], x[1, 4] = INF, 1.0
    x[2, 3], x[2, 4] = NAN, INF
    x[3, :4] = torch.tensor([2.0 ** -133, -2.0 ** -133, 0.0, 0.0], dtype=BF16)      # smallest subnormal
    x[4] = torch.finfo(BF16).max
    q, scale = torch.empty_like(x, dtype=E4M3), vec(5)
    B.quantize_rows(x, q, scale)
    assert scale[0] == 1 and torch.equal(q[0, :codes.numel()].float(), codes)
    assert scale[1] == INF and q[1, 3].float().isnan() and q[1, 4].float() == 0
    assert scale[2].isnan() and q[2].float().isnan().all()
    assert scale[3] > 0 and q[3, 0].float() > 400 and q[3, 1].float() < -400 and (q[3, 2:].float() == 0).all()
    assert (q[4].float() == 448).all()


# ----------------------------------------------------------------------------------------------- gated feed-forward ---

GATED_SHAPES = [(1, 1, 1), (1, 8, 8), (3, 5, 7), (2, 64, 64), (16, 64, 136), (5, 33, 130), (8, 1024, 200), (1, 4096, 1000), (31, 512, 96),
                (64, 72, 1032), (100, 200, 104), (127, 96, 200), (128, 128, 128), (129, 136, 264), (200, 48, 257), (257, 768, 520),
                (300, 72, 1032), (640, 256, 384), (1000, 136, 264), (1300, 2008, 1000), (1537, 1800, 904)]
GATED_LAYOUTS = [(0, 0), (8, 0), (0, 1)]


def product_tol(a, b, k):
    """Largest error of a float sum of k products: k 2^-23 of the sum of magnitudes."""
    return (k + 8) * 2.0 ** -23 * (a.double().abs() @ b.double().abs())


def check_gated_h(h, x64, wg64, wu64, kind, gate=None, up=None):
    g64, u64 = x64 @ wg64.T, x64 @ wu64.T
    eg, eu = product_tol(x64, wg64.T, x64.shape[1]), product_tol(x64, wu64.T, x64.shape[1])
    a64, _ = act_and_slope64(kind, g64)
    if gate is not None:
        close(gate, g64, U * 1.001 * g64.abs() + eg, "gate")
        close(up, u64, U * 1.001 * u64.abs() + eu, "up")
    # |a'| <= 1.13; a itself is evaluated to 2^-19 of its value (a few float operations) or of |g| (its tanh form)
    ea = 1.13 * eg + 2.0 ** -19 * g64.abs()
    close(h, a64 * u64, U * 1.001 * (a64 * u64).abs() + 1.01 * (ea * (u64.abs() + eu) + a64.abs() * eu), "h")


@pytest.mark.parametrize("tokens,width,ffn", GATED_SHAPES)
@pytest.mark.parametrize("pad,shift", GATED_LAYOUTS)
@pytest.mark.parametrize("kind", [B.ACT_SILU, B.ACT_GELU_TANH])
def test_gated_forward_and_backward_match_definition(tokens, width, ffn, pad, shift, kind):
    box = lambda r, c, data=None: Box(r, c, BF16, c + pad, shift, data)  # noqa: E731
    x = box(tokens, width, normal(1, tokens, width))
    wg, wu = (box(ffn, width, normal(s, ffn, width, std=1.5 / math.sqrt(width))) for s in (2, 3))
    h, gate, up = box(tokens, ffn), box(tokens, ffn), box(tokens, ffn)
    B.gated_ffn(x.t, wg.t, wu.t, h.t, gate=gate.t, up=up.t, activation=kind)
    check_gated_h(h.t, x.t.double(), wg.t.double(), wu.t.double(), kind, gate.t, up.t)
    alone = box(tokens, ffn)
    B.gated_ffn(x.t, wg.t, wu.t, alone.t, activation=kind)   # without the kept products: the same bits
    assert torch.equal(alone.t, h.t)
    # backward from the rounded gate and up
    dh = box(tokens, ffn, normal(4, tokens, ffn))
    dgate, dup, dx, dwg, dwu = box(tokens, ffn), box(tokens, ffn), box(tokens, width), box(ffn, width), box(ffn, width)
    B.gated_ffn_backward(dh.t, x.t, wg.t, wu.t, gate.t, up.t, dgate.t, dup.t, dx=dx.t, dw_gate=dwg.t, dw_up=dwu.t, activation=kind)
    a64, s64 = act_and_slope64(kind, gate.t.double())
    want_g, want_u = dh.t.double() * up.t.double() * s64, dh.t.double() * a64
    # a' and a are sums of a few terms of size up to 1 + |g|: 2^-19 of those, then one rounding
    size = 1 + gate.t.double().abs()
    close(dgate.t, want_g, U * 1.001 * want_g.abs() + 2.0 ** -19 * (dh.t.double() * up.t.double()).abs() * size, "dgate")
    close(dup.t, want_u, U * 1.001 * want_u.abs() + 2.0 ** -19 * dh.t.double().abs() * size, "dup")
    # the products take dgate and dup as they are stored
    dg, du, x64 = dgate.t.double(), dup.t.double(), x.t.double()
    want = dg @ wg.t.double() + du @ wu.t.double()
    tol = product_tol(dg, wg.t, 2 * ffn) + product_tol(du, wu.t, 2 * ffn)
    close(dx.t, want, U * 1.001 * want.abs() + tol, "dx")
    for got, d in ((dwg, dg), (dwu, du)):
        want = d.T @ x64
        close(got.t, want, U * 1.001 * want.abs() + product_tol(d.T, x64, tokens), "dw")
    for b in (x, wg, wu, h, gate, up, dh, dgate, dup, dx, dwg, dwu):
        assert b.untouched_outside()
    # one output at a time, dgate and dup in the place of gate and up: the same bits
    only, og, ou = box(tokens, width), box(ffn, width), box(ffn, width)
    B.gated_ffn_backward(dh.t, None, wg.t, wu.t, gate.t, up.t, dgate.t, dup.t, dx=only.t, activation=kind)
    B.gated_ffn_backward(dh.t, x.t, None, None, gate.t, up.t, gate.t, up.t, dw_gate=og.t, dw_up=ou.t, activation=kind)
    assert torch.equal(only.t, dx.t) and torch.equal(og.t, dwg.t) and torch.equal(ou.t, dwu.t)
    assert torch.equal(gate.t, dgate.t) and torch.equal(up.t, dup.t)


@pytest.mark.parametrize("tokens,width,ffn", GATED_SHAPES + [(16, 256, 512), (130, 1040, 272), (1300, 272, 1040), (1793, 4096, 800)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (16, 0), (0, 1)])
def test_gated_8_bits_matches_definition(tokens, width, ffn, pad, shift):
    def rows8(seed, rows, std):
        q, scale = Box(rows, width, E4M3, width + pad, shift), vec(rows)
        B.quantize_rows(normal(seed, rows, width, std=std), q.t, scale)
        return q, scale, q.t.double() * scale.double()[:, None]
    x, sx, x64 = rows8(1, tokens, 1.0)
    wg, sg, wg64 = rows8(2, ffn, 1.5 / math.sqrt(width))
    wu, su, wu64 = rows8(3, ffn, 1.5 / math.sqrt(width))
    for kind in (B.ACT_SILU, B.ACT_GELU_TANH):
        h = Box(tokens, ffn, BF16, ffn + pad, shift)
        B.gated_ffn_e4m3(x.t, sx, wg.t, sg, wu.t, su, h.t, kind)
        check_gated_h(h.t, x64, wg64, wu64, kind)
        assert h.untouched_outside()


def test_gated_views_of_one_buffer_and_three_dimensions():
    # gate and up as the halves of one [tokens, 2 ffn] buffer, the weights as the halves of one [2 ffn, width] buffer
    b, t, width, ffn = 2, 75, 128, 192
    x = normal(1, b, t, width)
    w = normal(2, 2 * ffn, width, std=0.1)
    both, h = torch.zeros(b, t, 2 * ffn, dtype=BF16, device="cuda"), torch.zeros(b, t, ffn, dtype=BF16, device="cuda")
    B.gated_ffn(x, w[:ffn], w[ffn:], h, gate=both[..., :ffn], up=both[..., ffn:])
    flat = both.view(-1, 2 * ffn)
    check_gated_h(h.view(-1, ffn), x.view(-1, width).double(), w[:ffn].double(), w[ffn:].double(), 0, flat[:, :ffn], flat[:, ffn:])


def test_gated_rows_do_not_mix():
    # a token of NaNs or infinities stays in its own row, forward and in dx
    tokens, width, ffn = 140, 64, 96
    x, wg, wu, dh = normal(1, tokens, width), normal(2, ffn, width), normal(3, ffn, width), normal(4, tokens, ffn)
    new = lambda *s: torch.zeros(s, dtype=BF16, device="cuda")  # noqa: E731

    def both():
        h, gate, up, dx, dg, du = new(tokens, ffn), new(tokens, ffn), new(tokens, ffn), new(tokens, width), new(tokens, ffn), new(tokens, ffn)
        B.gated_ffn(x, wg, wu, h, gate=gate, up=up)
        B.gated_ffn_backward(dh, None, wg, wu, gate, up, dg, du, dx=dx)
        return h, dx
    clean = both()
    x[77, 5], x[139] = NAN, INF
    dh[3, 1] = NAN
    dirty = both()
    keep = torch.ones(tokens, dtype=torch.bool, device="cuda")
    keep[77] = keep[139] = False
    assert torch.equal(clean[0][keep], dirty[0][keep]) and dirty[0][77].isnan().all()
    keep[3] = False
    assert torch.equal(clean[1][keep], dirty[1][keep]) and dirty[1][3].isnan().all() and dirty[1][77].isnan().all()


def test_activation_at_the_ends_of_the_range():
    # width 1, weights 1: the products are the values themselves
    g = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 5.0, -5.0, 20.0, -20.0, 88.0, -88.0, 104.0, -104.0, 1e4, -1e4, 1e30, -1e30, 3e38, -3e38],
                     dtype=BF16, device="cuda")[:, None]
    one = torch.ones(1, 1, dtype=BF16, device="cuda")
    n = g.shape[0]
    for kind in (B.ACT_SILU, B.ACT_GELU_TANH):
        w8 = torch.zeros(n, 8, dtype=BF16, device="cuda")
        w8[:, :1] = g
        for x, wg in ((g, one), (w8, torch.nn.functional.pad(one, (0, 7)))):           # unaligned and aligned rows
            gate, up, h = (torch.zeros(n, 1, dtype=BF16, device="cuda") for _ in range(3))
            ones = torch.ones(n, 1, dtype=BF16, device="cuda")
            B.gated_ffn(x, wg, wg, h, gate=gate, up=up, activation=kind)
            assert torch.equal(gate, g) and torch.equal(up, g)
            dg, du = torch.zeros_like(h), torch.zeros_like(h)
            B.gated_ffn_backward(ones, None, wg, wg, gate, ones, dg, du, dx=torch.zeros_like(x), activation=kind)
            small = g.abs() < 1e15                          # g^3 stays finite in 64 and the slope's terms in 32 bits
            a, s = act_and_slope64(kind, g.double())
            close(du[small], a[small], (U * 1.001 * a.abs() + 2.0 ** -19 * (1 + g.double().abs()) * 2.0 ** -3)[small], "a")
            close(dg[small], s[small], (U * 1.001 + 2.0 ** -19 * (1 + g.double().abs().clamp_max(1e3)))[small], "slope")
            assert not h.isnan().any() and not du.isnan().any() and not dg.isnan().any()


def test_gated_gradient_agrees_with_differences():
    tokens, width, ffn = 3, 8, 16
    for kind in (B.ACT_SILU, B.ACT_GELU_TANH):
        x, wg, wu, dh = normal(1, tokens, width), normal(2, ffn, width), normal(3, ffn, width), normal(4, tokens, ffn)
        new = lambda *s: torch.zeros(s, dtype=BF16, device="cuda")  # noqa: E731
        h, gate, up = new(tokens, ffn), new(tokens, ffn), new(tokens, ffn)
        dx, dwg, dwu = new(tokens, width), new(ffn, width), new(ffn, width)
        B.gated_ffn(x, wg, wu, h, gate=gate, up=up, activation=kind)
        B.gated_ffn_backward(dh, x, wg, wu, gate, up, new(tokens, ffn), new(tokens, ffn), dx=dx, dw_gate=dwg, dw_up=dwu, activation=kind)
        args = [x.double(), wg.double(), wu.double()]

        def objective(x, wg, wu):
            return (dh.double() * act_and_slope64(kind, x @ wg.T)[0] * (x @ wu.T)).sum()
        for which, grad in enumerate((dx, dwg, dwu)):
            want, step = torch.zeros_like(args[which]), 1e-5
            for i in range(want.numel()):
                e = torch.zeros(want.numel(), dtype=torch.float64, device="cuda")
                e[i] = step
                p, m = list(args), list(args)
                p[which], m[which] = args[which] + e.view_as(want), args[which] - e.view_as(want)
                want.view(-1)[i] = (objective(*p) - objective(*m)) / (2 * step)
            # gate, up, dgate, dup and the result are each rounded once: relative to the size of the terms, below 5 U of their
            # root sum of squares, here bounded by 5 U of the largest entry
            assert (grad.double() - want).abs().max() <= 5 * U * want.abs().max()


def test_empty_extents():
    new = lambda *s: torch.full(s, 7.0, dtype=BF16, device="cuda")  # noqa: E731
    ws = torch.zeros(B.rms_norm_workspace_bytes(16), dtype=torch.uint8, device="cuda")
    dw = new(16)
    B.add_rms_norm(new(0, 16), new(0, 16), new(16), EPS, residual_out=new(0, 16), y=new(0, 16))
    B.add_rms_norm_backward(new(0, 16), new(0, 16), vec(0), new(16), new(0, 16), dw, ws)
    assert (dw == 0).all()                                  # the sum over no rows
    scale = vec(3)
    B.quantize_rows(new(3, 0), torch.empty(3, 0, dtype=E4M3, device="cuda"), scale)
    assert (scale == 0).all()
    h = new(4, 8)
    B.gated_ffn(new(4, 0), new(8, 0), new(8, 0), h)
    assert (h == 0).all()                                   # sums over no terms
    B.gated_ffn(new(0, 16), new(8, 16), new(8, 16), new(0, 8), gate=new(0, 8), up=new(0, 8))
    dwg, dwu, dx = new(8, 16), new(8, 16), new(0, 16)
    B.gated_ffn_backward(new(0, 8), new(0, 16), new(8, 16), new(8, 16), new(0, 8), new(0, 8), new(0, 8), new(0, 8), dx=dx, dw_gate=dwg, dw_up=dwu)
    assert (dwg == 0).all() and (dwu == 0).all()
    dx = new(4, 16)
    B.gated_ffn_backward(new(4, 0), None, new(0, 16), new(0, 16), new(4, 0), new(4, 0), new(4, 0), new(4, 0), dx=dx)
    assert (dx == 0).all()
    e = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    z, loss, dz = normal(1, 3, 50), vec(3), new(3, 50)
    B.distill_loss_and_grad(z, e, torch.empty(3, 0, device="cuda"), 1.0, torch.ones(3, device="cuda"), loss, dz)
    assert (loss == 0).all() and (dz == 0).all()            # a teacher without entries
    B.distill_loss(z[:0], e[:0], torch.empty(0, 0, device="cuda"), 1.0, vec(0))


# ----------------------------------------------------------------------------------------------------- distillation ---

def teacher(seed, rows, vocab, k, index=torch.int64, distinct=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if distinct:
        at = torch.rand(rows, vocab, generator=g, device="cuda").topk(k, dim=1).indices
    else:
        at = torch.randint(0, vocab, (rows, k), generator=g, device="cuda")
    return at.to(index), torch.randn(rows, k, generator=g, device="cuda") * 3


def check_distill(z, at, top, tau, weight=None, box_args=None, what=""):
    rows, vocab = z.shape
    weight = torch.ones(rows, device="cuda") if weight is None else weight
    loss64, lse64, grad64 = distill64(z, at, top, tau)
    zero = weight == 0
    want = torch.where(zero[:, None], 0.0, grad64 * weight.double()[:, None])
    finite = z.double()[z.isfinite()]
    spread = (finite.max() - finite.min()).item() / tau + 20 if finite.numel() else 20.0
    # exp of an argument up to `spread` in size: spread 2^-23 + 2^-21 of the value; its sums: (vocab / 64 + 16) 2^-23
    rel = spread * 2.0 ** -22 + 2.0 ** -20 + (vocab / 64 + 16) * 2.0 ** -23
    q = torch.softmax(z.double() / tau, 1)
    tol = rel * 4 * tau * weight.double().abs()[:, None] * (q + (want / (tau * weight.double()[:, None])).nan_to_num().abs() + 2.0 ** -30)
    if z.dtype == BF16:
        tol = tol + U * 1.001 * want.abs()
    ltol = 4 * tau * tau * (rel + spread * 2.0 ** -22)
    pad, shift = box_args or (0, 0)
    out = Box(rows, vocab, z.dtype, vocab + pad, shift)
    loss, lse = vec(rows), vec(rows)
    B.distill_loss(z, at, top, tau, loss, lse=lse)
    close(loss, loss64, ltol, what + " loss")
    close(lse, lse64, 2 * rel + 2.0 ** -22 * lse64.nan_to_num(0, 0, 0).abs(), what + " lse")
    bare = vec(rows)
    B.distill_loss(z, at, top, tau, bare)
    assert torch.equal(bare.nan_to_num(-7.0), loss.nan_to_num(-7.0))
    B.distill_loss_backward(z, at, top, tau, lse, weight, out.t)
    close(out.t, want, tol, what + " dlogits (backward)")
    assert out.untouched_outside()
    both, fused = Box(rows, vocab, z.dtype, vocab + pad, shift), vec(rows)
    B.distill_loss_and_grad(z, at, top, tau, weight, fused, both.t)
    close(both.t, want, tol, what + " dlogits (one pass)")
    close(fused, torch.where(zero, 0.0, weight.double() * loss64), ltol * weight.double().abs(), what + " weighted loss")
    assert both.untouched_outside()
    place = Box(rows, vocab, z.dtype, vocab + pad, shift, z)
    B.distill_loss_and_grad(place.t, at, top, tau, weight, fused, place.t)       # over the logits themselves
    close(place.t, want, tol, what + " dlogits (in place)")
    place.t.copy_(z)
    B.distill_loss_backward(place.t, at, top, tau, lse, weight, place.t)
    close(place.t, want, tol, what + " dlogits (backward in place)")
    assert place.untouched_outside()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 2, 2), (3, 17, 5), (5, 1000, 16), (4, 4099, 100), (3, 32000, 64), (9, 50257, 21),
                                          (2, 65544, 8), (2, 131072, 257), (1, 200_003, 1024), (2, 900_001, 4), (600, 300, 7),
                                          (1300, 1030, 33), (500, 5001, 12), (450, 17_003, 20)])
def test_distill_matches_definition(rows, vocab, k, dtype):
    z = normal(rows + vocab, rows, vocab, std=2.0, dtype=dtype)
    at, top = teacher(1, rows, vocab, k)
    check_distill(z, at, top, 1.0)
    weight = torch.linspace(-0.5, 1.5, rows, device="cuda") if rows > 1 else torch.full((1,), 0.3, device="cuda")
    at, top = teacher(2, rows, vocab, k, torch.int32, distinct=False)            # indexes that appear more than once
    check_distill(z, at, top, 2.5, weight)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("vocab", [1031, 50_000])
def test_distill_strided_logits(dtype, pad, shift, vocab):
    rows, k = 6, 12
    z = Box(rows, vocab, dtype, vocab + pad, shift, normal(7, rows, vocab, std=2.0, dtype=dtype))
    at, top = teacher(3, rows, vocab, k)
    wide_at, wide_top = torch.full((rows, k + 3), -5, device="cuda"), torch.zeros(rows, k + 1, device="cuda")
    wide_at[:, :k], wide_top[:, :k] = at, top
    check_distill(z.t, wide_at[:, :k], wide_top[:, :k], 1.5, box_args=(pad, shift))
    check_distill(z.t, at, top, 1.5, box_args=(0, 2))                             # logits and gradient aligned differently
    assert z.untouched_outside()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [700, 33_001])
def test_distill_absent_entries_masks_and_non_finite_rows(dtype, vocab):
    rows, k = 12, 9
    z = normal(11, rows, vocab, std=2.0, dtype=dtype)
    at, top = teacher(5, rows, vocab, k)
    at[0, 4:] = -1                                           # fewer entries than k
    at[1] = -1                                               # none
    at[2, 0], at[2, 1] = vocab, 2 ** 40                      # not in the vocabulary
    top[3, 2:] = -INF                                        # entries without mass
    top[4] = -INF
    z[5] = NAN                                               # a row that weighs nothing
    z[6] = NAN                                               # a row without entries
    at[6] = -1
    gone = torch.ones(vocab, dtype=torch.bool, device="cuda")
    gone[at[7]] = False
    z[7, gone.nonzero()[: vocab // 2, 0]] = -INF             # masked columns that the teacher does not want
    z[8, at[8, 0]] = -INF                                    # one that it does want: infinite loss, finite gradient
    z[9] = torch.finfo(dtype).min                            # a row of the type's lowest value: uniform
    z[10, vocab // 2:] = torch.finfo(dtype).min
    top[11, 3] = top[11, 3] + 300                            # one entry has all the mass
    weight = torch.full((rows,), 0.25, device="cuda")
    weight[5] = 0
    loss, lse, dz = vec(rows), vec(rows), torch.zeros_like(z)
    B.distill_loss_and_grad(z, at, top, 1.0, weight, loss, dz)
    for i in (1, 4, 5, 6):
        assert loss[i] == 0 and (dz[i] == 0).all(), i
    assert loss[8] == INF and dz[8].isfinite().all()
    want = torch.full((vocab,), 0.25 / vocab, dtype=torch.float64, device="cuda")
    p = torch.softmax(top[9].double(), 0)
    want[at[9]] -= 0.25 * p
    close(dz[9], want, U * 1.01 * want.abs() + 1e-6, "uniform row")
    ok = torch.tensor([0, 1, 2, 3, 4, 7, 10, 11], device="cuda")
    want = 0.25 * distill64(z[ok], at[ok], top[ok], 1.0)[0]                       # row 10 wants masked columns: about 1e37, so in relative terms
    close(loss[ok], want, 1e-4 + 2.0 ** -18 * want.abs(), "losses")
    check = [0, 1, 2, 3, 4, 7, 11]
    check_distill(z[check], at[check], top[check], 1.0, weight[check])
    B.distill_loss(z, at, top, 1.0, loss, lse=lse)
    assert loss[5].isnan() and loss[6] == 0 and lse[6].isnan()
    B.distill_loss_backward(z, at, top, 1.0, lse, weight, dz)
    assert (dz[5] == 0).all() and (dz[6] == 0).all() and (dz[1] == 0).all() and dz[8].isfinite().all()
    # all of a row's logits -infinity, or one of them +infinity: no distribution
    z[0] = -INF
    z[1, 0], at[1, 0] = INF, 1
    B.distill_loss_and_grad(z[:2], at[:2], top[:2], 1.0, weight[:2], loss[:2], dz[:2])
    assert loss[:2].isnan().all() and dz[0].isnan().all() and dz[1, 0].isnan()
    # a NaN among the teacher's logits
    top[2, 5] = NAN
    B.distill_loss_and_grad(z[2:3], at[2:3], top[2:3], 1.0, weight[2:3], loss[2:3], dz[2:3])
    assert loss[2].isnan()


def test_distill_gradient_agrees_with_differences():
    rows, vocab, k, tau = 2, 40, 6, 1.7
    z = normal(1, rows, vocab, std=2.0, dtype=F32)
    at, top = teacher(2, rows, vocab, k, distinct=False)
    loss, dz = vec(rows), torch.zeros_like(z)
    B.distill_loss_and_grad(z, at, top, tau, torch.ones(rows, device="cuda"), loss, dz)
    for i in range(rows):
        for j in range(vocab):
            e = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda")
            e[i, j] = 1e-5
            d = (distill64(z.double() + e, at, top, tau)[0][i] - distill64(z.double() - e, at, top, tau)[0][i]) / 2e-5
            assert abs(d.item() - dz[i, j].item()) <= 1e-5


# ------------------------------------------------------------------------------- streams, graphs, repetition, offsets ---

def one_of_each(stream=None, seed=0, tokens=70, width=256, ffn=320, vocab=5003, k=7):
    """All operators once on fixed inputs; returns the launch closure and its outputs."""
    new = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    x, res, w = normal(seed, tokens, width), normal(seed + 1, tokens, width), normal(seed + 2, width)
    wg, wu, dh = normal(seed + 3, ffn, width, std=0.1), normal(seed + 4, ffn, width, std=0.1), normal(seed + 5, tokens, ffn)
    z = normal(seed + 6, tokens, vocab, std=2.0)
    at, top = teacher(seed + 7, tokens, vocab, k)
    weight = torch.ones(tokens, device="cuda")
    o = dict(r=new(tokens, width), y=new(tokens, width), y8=new(tokens, width, dtype=E4M3), s8=new(tokens, dtype=F32), rstd=new(tokens, dtype=F32),
             g8=new(ffn, width, dtype=E4M3), gs=new(ffn, dtype=F32), u8=new(ffn, width, dtype=E4M3), us=new(ffn, dtype=F32), h8=new(tokens, ffn),
             h=new(tokens, ffn), gate=new(tokens, ffn), up=new(tokens, ffn), dg=new(tokens, ffn), du=new(tokens, ffn), dy=new(tokens, width),
             dwg=new(ffn, width), dwu=new(ffn, width), dx=new(tokens, width), dw=new(width), loss=new(tokens, dtype=F32), dz=new(tokens, vocab),
             l2=new(tokens, dtype=F32), lse=new(tokens, dtype=F32), dz2=new(tokens, vocab))
    ws = torch.zeros(B.rms_norm_workspace_bytes(width), dtype=torch.uint8, device="cuda")

    def launch(s=stream):
        B.add_rms_norm(x, res, w, EPS, residual_out=o["r"], y=o["y"], y8=o["y8"], y8_scale=o["s8"], rstd=o["rstd"], stream=s)
        B.quantize_rows(wg, o["g8"], o["gs"], stream=s)
        B.quantize_rows(wu, o["u8"], o["us"], stream=s)
        B.gated_ffn_e4m3(o["y8"], o["s8"], o["g8"], o["gs"], o["u8"], o["us"], o["h8"], stream=s)
        B.gated_ffn(o["y"], wg, wu, o["h"], gate=o["gate"], up=o["up"], stream=s)
        B.gated_ffn_backward(dh, o["y"], wg, wu, o["gate"], o["up"], o["dg"], o["du"], dx=o["dy"], dw_gate=o["dwg"], dw_up=o["dwu"], stream=s)
        B.add_rms_norm_backward(o["dy"], o["r"], o["rstd"], w, o["dx"], o["dw"], ws, dresidual=res, stream=s)
        B.distill_loss_and_grad(z, at, top, 2.0, weight, o["loss"], o["dz"], stream=s)
        B.distill_loss(z, at, top, 2.0, o["l2"], lse=o["lse"], stream=s)
        B.distill_loss_backward(z, at, top, 2.0, o["lse"], weight, o["dz2"], stream=s)
    return launch, o


def bits_of(outputs):
    torch.cuda.synchronize()
    return {k: v.contiguous().view(torch.uint8).clone() for k, v in outputs.items()}


def test_repeated_calls_side_streams_and_graphs_give_the_same_bits():
    launch, o = one_of_each()
    launch()
    first = bits_of(o)
    assert all(v.any() for v in first.values())
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    for how in ("again", "side", "graph"):
        for v in o.values():
            v.view(torch.uint8).zero_()
        torch.cuda.synchronize()
        if how == "again":
            launch()
        elif how == "side":
            launch(side)
        else:
            with torch.cuda.graph(graph):
                launch(torch.cuda.current_stream())
            graph.replay()
        now = bits_of(o)
        assert B.pipeline_fault() == 0
        assert all(torch.equal(first[k], now[k]) for k in first), how
    del graph


def test_offsets_beyond_32_bits():
    # four rows 2^31 elements apart: the last one begins 3 * 2^31 elements into the buffer (17 GB of bfloat16)
    ld = 1 << 31
    big = torch.empty(3 * ld + 4096, dtype=BF16, device="cuda")
    rows, width, ffn = 4, 256, 384
    x = big.as_strided((rows, width), (ld, 1), 0)
    y = big.as_strided((rows, width), (ld, 1), 512)
    h = big.as_strided((rows, ffn), (ld, 1), 1024)
    x.copy_(normal(1, rows, width))
    weight = normal(2, width)
    B.add_rms_norm(x, None, weight, EPS, y=y)
    want = x.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + EPS) * weight.double()
    close(y, want, U * 1.01 * want.abs(), "norm")
    wg, wu = normal(3, ffn, width, std=0.1), normal(4, ffn, width, std=0.1)
    B.gated_ffn(y, wg, wu, h)
    check_gated_h(h, y.double(), wg.double(), wu.double(), 0)
    z, dz = big.as_strided((rows, 1000), (ld, 1), 2048), big.as_strided((rows, 1000), (ld, 1), 3056)
    z.copy_(normal(5, rows, 1000, std=2.0))
    at, top = teacher(6, rows, 1000, 5)
    loss = vec(rows)
    B.distill_loss_and_grad(z, at, top, 1.0, torch.ones(rows, device="cuda"), loss, dz)
    loss64, _, grad64 = distill64(z, at, top, 1.0)
    close(loss, loss64, 1e-4, "loss")
    close(dz, grad64, U * 1.01 * grad64.abs() + 1e-6, "dlogits")


def test_the_binding_refuses_what_it_cannot_describe():
    x, w = normal(1, 4, 64), normal(2, 64)
    y, rstd = torch.empty_like(x), vec(4)

    def refused(f, *a, status=B.ERR_ARG, **k):
        with pytest.raises(B.CollageError) as e:
            f(*a, **k)
        assert e.value.status == status
    refused(B.add_rms_norm, x.float(), None, w, EPS, y=y)                         # type
    refused(B.add_rms_norm, x.cpu(), None, w, EPS, y=y)                           # device
    refused(B.add_rms_norm, x.t(), None, w, EPS, y=y)                             # columns not contiguous
    refused(B.add_rms_norm, x[0], None, w, EPS, y=y)                              # one dimension
    refused(B.add_rms_norm, x, None, w[:32], EPS, y=y)                            # weight's length
    refused(B.add_rms_norm, x, None, w, EPS, y=y[:, :32])                         # shapes
    refused(B.add_rms_norm, x, None, w, EPS, y=y, rstd=rstd[:3])
    refused(B.add_rms_norm, x, None, w, EPS, status=B.ERR_NULL)                   # no output
    refused(B.add_rms_norm, None, None, w, EPS, y=y, status=B.ERR_NULL)
    refused(B.add_rms_norm, normal(1, 2, 3, 64).transpose(0, 1), None, w, EPS, y=y)     # rows of no single stride
    refused(B.quantize_rows, x, torch.empty_like(x), vec(4))
    refused(B.gated_ffn, x, normal(1, 8, 64), normal(1, 8, 32), torch.zeros(4, 8, dtype=BF16, device="cuda"))
    square = normal(1, 64, 64)
    refused(B.gated_ffn, square, square, square, square, status=B.ERR_ALIAS)
    at, top = teacher(1, 4, 64, 3)
    refused(B.distill_loss, x.half(), at, top, 1.0, vec(4))
    refused(B.distill_loss, x, at.short(), top, 1.0, vec(4))
    refused(B.distill_loss, x, at, top, 0.0, vec(4))
    refused(B.distill_loss, x, at, top, 1.0, None, status=B.ERR_NULL)
