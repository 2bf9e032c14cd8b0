"""Norms around a block against their definition in 64 bits, forward and backward.

Tolerances.  One rounding to bfloat16 is at most U = 2^-8 of the value.  A float sum of K terms, split over at least 32 threads, is at
most (K / 32 + 16) 2^-23 of the sum of their magnitudes off (`deep`).  Products, sums and the gate's exponential (a few units of a
float's last place for the gates' size here, at most 6) are within 2^-20 (`E`) of the magnitudes that go in.
"""
import math

import pytest
import torch

from ops_util import BF16, E4M3, F32, U, Box, close, normal
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS, E = 1e-6, 2.0 ** -20
INF, NAN = math.inf, math.nan

SHAPES = [(1, 1), (3, 7), (2, 8), (5, 64), (33, 257), (7, 768), (3, 1000), (130, 1024), (1, 4096), (19, 4096), (9, 5120), (3, 8192), (2, 11008),
          (5, 16384), (2, 20008), (2, 40003)]
MANY = [(300, 64), (1025, 136), (301, 520), (700, 1024), (310, 257), (400, 4096), (299, 8192), (330, 16384), (299, 5120)]
LAYOUTS = [(0, 0), (8, 0), (3, 0), (0, 1)]              # (row stride beyond the columns, elements off a 16-byte boundary)
FORMS = [("channel", B.GATE_NONE, True, True), ("token", B.GATE_SIGMOID, True, True), ("none", B.GATE_NONE, True, True),
         ("channel", B.GATE_SILU, False, True), ("token", B.GATE_SILU, True, False), ("channel", B.GATE_SIGMOID, True, False), ("none", B.GATE_NONE, False, False)]
ALPHA, BETA = 0.9, -0.3


def vec(n, dtype=F32):
    return torch.full((n,), NAN, dtype=F32, device="cuda").to(dtype)


def gate64(kind, g):
    """The gate's value, its slope, and a bound of the magnitudes that went into the slope."""
    if kind == B.GATE_NONE:
        return g, torch.ones_like(g), torch.ones_like(g)
    s = torch.sigmoid(g)
    if kind == B.GATE_SIGMOID:
        return s, s * torch.sigmoid(-g), s
    return g * s, s + g * s * torch.sigmoid(-g), s + (g * s).abs()


class Case:
    def __init__(self, rows, cols, pad, shift, form, seed=0, gate_rows=None):
        self.rows, self.cols, (self.gate_kind, self.act, self.post_on, self.pre_on) = rows, cols, form
        self.box = lambda dtype=BF16, data=None, n=rows: Box(n, cols, dtype, cols + pad, shift, data)
        self.x, self.o = self.box(data=normal(seed, rows, cols, std=3.0)), self.box(data=normal(seed + 1, rows, cols))
        n = {"none": None, "channel": 1, "token": rows}[self.gate_kind]
        self.gate = None if n is None else self.box(data=normal(seed + 2, n, cols, std=2.0), n=n)
        self.post = normal(seed + 3, cols) if self.post_on else None
        self.pre = normal(seed + 4, cols) if self.pre_on else None
        self.kw = dict(gate=self.gate and self.gate.t, post_weight=self.post, pre_weight=self.pre, residual_scale=ALPHA, block_scale=BETA, activation=self.act)
        self.A, self.slope, self.slope_mag = (1.0, None, None) if self.gate is None else gate64(self.act, self.gate.t.double())


def check_forward(case, out8=True, in_place=None):
    rows, cols, c = case.rows, case.cols, case
    x64, o64 = c.x.t.double(), c.o.t.double()
    r, y, y8 = c.box(), c.box() if c.pre_on else None, c.box(E4M3) if out8 and c.pre_on else None
    if in_place == "x":
        r = c.x
    elif in_place == "block":
        r = c.o
    elif in_place == "y" and c.pre_on:
        y = c.o
    scale, rpost, rpre = (vec(rows) if on else None for on in (y8, c.post_on, c.pre_on))
    B.block_norm(c.x.t, c.o.t, r.t, y=y and y.t, y8=y8 and y8.t, y8_scale=scale, rstd_post=rpost, rstd_pre=rpre, eps=EPS, **c.kw)
    deep = (cols / 32 + 16) * 2.0 ** -23
    n = o64
    if c.post_on:
        rstd = 1 / torch.sqrt((o64 * o64).mean(1, keepdim=True) + EPS)
        close(rpost, rstd[:, 0], (deep + E) * rstd[:, 0], "rstd_post")
        n = o64 * rstd * c.post.double()
    added = BETA * c.A * n
    r64, size = ALPHA * x64 + added, (ALPHA * x64).abs() + added.abs()
    off = size * (deep + E)                             # of r in float
    close(r.t, r64, U * 1.001 * r64.abs() + 1.01 * off, "r")
    if c.pre_on:
        rms = torch.sqrt((r64 * r64).mean(1, keepdim=True) + EPS)
        rel = deep + E + 1.01 * torch.sqrt((off * off).mean(1, keepdim=True)) / rms      # of 1 / rms
        close(rpre, 1 / rms[:, 0], (rel / rms)[:, 0], "rstd_pre")
        w = c.pre.double()
        y64 = r64 / rms * w
        y_off = y64.abs() * (rel + E) + (w / rms).abs() * off
        if y is not None:
            close(y.t, y64, U * 1.001 * y64.abs() + 1.01 * y_off, "y")
        if y8 is not None:
            scale64, most = y64.abs().amax(1), y_off.amax(1)
            close(scale, scale64 / 448, 1.01 * (most + E * scale64) / 448, "scale")
            step = scale64[:, None] / 448 * 2.0 ** -10 * 1.001
            close(y8.t.double() * scale.double()[:, None], y64, y64.abs() * (2.0 ** -4 + E) + step + 1.2 * y_off + 1.01 * (y64.abs() / scale64.clamp_min(1e-300)[:, None]) * most[:, None], "y8")
    for b in (c.x, c.o, c.gate, r, y, y8):
        assert b is None or b.untouched_outside()


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad,shift", LAYOUTS)
def test_forward_matches_definition(rows, cols, pad, shift):
    for i, form in enumerate(FORMS):
        check_forward(Case(rows, cols, pad, shift, form, seed=10 * i), out8=i % 2 == 0)


@pytest.mark.parametrize("rows,cols", MANY)
def test_forward_of_many_rows(rows, cols):
    check_forward(Case(rows, cols, 0, 0, FORMS[0]))
    check_forward(Case(rows, cols, 8, 0, FORMS[1], seed=3))


@pytest.mark.parametrize("place", ["x", "block", "y"])
@pytest.mark.parametrize("rows,cols", [(5, 64), (3, 1001), (3, 4096), (2, 40000)])
def test_forward_in_place(rows, cols, place):
    for form in FORMS[:3]:
        check_forward(Case(rows, cols, 0, 0, form), in_place=place)


def check_backward(case, use_dy=True, use_dr=True, seed=50):
    c, rows, cols = case, case.rows, case.cols
    use_dy = use_dy and c.pre_on
    dy, dr, r = c.box(data=normal(seed, rows, cols)), c.box(data=normal(seed + 1, rows, cols)), c.box(data=normal(seed + 2, rows, cols, std=2.0))
    rpost = (1 / torch.sqrt((c.o.t.double() ** 2).mean(1) + EPS)).float() if c.post_on else None
    rpre = (1 / torch.sqrt((r.t.double() ** 2).mean(1) + EPS)).float() if c.pre_on else None
    deep = (cols / 32 + 16) * 2.0 ** -23
    rows_deep = (rows + 16) * 2.0 ** -23
    D, D_size, D_off = 0, 0, 0
    if use_dy:
        rs = rpre.double()[:, None]
        nr, q = r.t.double() * rs, dy.t.double() * c.pre.double()
        mean, spread = (q * nr).mean(1, keepdim=True), (q * nr).abs().mean(1, keepdim=True)
        D = rs * (q - nr * mean)
        D_size = rs * (q.abs() + (nr * mean).abs())
        D_off = rs * nr.abs() * spread * deep
    if use_dr:
        D, D_size = D + dr.t.double(), D_size + dr.t.double().abs()
    D_off = D_off + E * D_size
    u, u_off = BETA * D, abs(BETA) * (D_off + E * D.abs())
    A = c.A if c.gate is not None else torch.ones(1, 1, dtype=torch.float64, device="cuda")
    du, du_off = u * A, A.abs() * (u_off + E * u.abs())
    rs_o = rpost.double()[:, None] if c.post_on else 1.0
    no, w = c.o.t.double() * rs_o, c.post.double() if c.post_on else torch.ones(cols, dtype=torch.float64, device="cuda")
    want, tol = {}, {}

    def expect(name, v, off):
        want[name], tol[name] = v, U * 1.001 * v.abs() + 1.02 * off + 1e-38
    expect("dx", ALPHA * D, ALPHA * (D_off + E * D.abs()))
    if c.post_on:
        h, h_off = du * w, w.abs() * (du_off + E * du.abs())
        mean, spread = (h * no).mean(1, keepdim=True), (h * no).abs().mean(1, keepdim=True)
        expect("dblock", rs_o * (h - no * mean), rs_o * (h_off + E * h.abs() + no.abs() * ((h_off * no.abs()).mean(1, keepdim=True) + spread * (deep + E))))
        expect("dpost_weight", (du * no).sum(0), ((du_off + E * du.abs()) * no.abs()).sum(0) + rows_deep * (du * no).abs().sum(0))
    else:
        expect("dblock", du, du_off)
    if use_dy:
        expect("dpre_weight", (dy.t.double() * nr).sum(0), (rows_deep + E) * (dy.t.double() * nr).abs().sum(0))
    if c.gate is not None:
        un, un_off = u * no * w, (u_off + E * u.abs()) * (no * w).abs()
        if c.gate.rows == 1 and rows > 1:
            s, s_off = un.sum(0, keepdim=True), un_off.sum(0, keepdim=True) + rows_deep * un.abs().sum(0, keepdim=True)
            expect("dgate", s * c.slope, s_off * c.slope_mag + 2 * E * s.abs() * c.slope_mag)
        else:
            expect("dgate", un * c.slope, un_off * c.slope_mag + 2 * E * un.abs() * c.slope_mag)
    ws = torch.full((B.block_norm_workspace_bytes(cols),), 0xFF, dtype=torch.uint8, device="cuda")

    def outputs(names):
        out = {}
        for k in names:
            out[k] = vec(cols, BF16) if k in ("dpost_weight", "dpre_weight") else c.box(n=c.gate.rows if k == "dgate" else rows)
        return out

    def call(out, dy_t=dy.t, dr_t=dr.t):
        t = {k: v.t if isinstance(v, Box) else v for k, v in out.items()}
        B.block_norm_backward(dy_t if use_dy else None, r.t if use_dy else None, c.o.t, rpost, rpre if use_dy else None, t.pop("dx", None), t.pop("dblock", None),
                              dr=dr_t if use_dr else None, workspace=ws, **c.kw, **t)
        return {k: v.t if isinstance(v, Box) else v for k, v in out.items()}
    whole = outputs(want)
    got = call(whole)
    for k in want:
        close(got[k], want[k], tol[k], k)
        assert not isinstance(whole[k], Box) or whole[k].untouched_outside()
    for k in want:                                       # one output at a time gives the same bits
        assert torch.equal(call(outputs([k]))[k], got[k]), k
    # gradients in the place of those that came in
    place = {k: v for k, v in outputs(want).items() if k not in ("dx", "dblock")}
    p, q = c.box(data=dy.t), c.box(data=dr.t)
    if use_dy and use_dr:
        also = call({**place, "dx": q, "dblock": p}, p.t, q.t)
    elif use_dr:
        also = call({**place, "dx": q}, None, q.t)
    else:
        also = call({**place, "dblock": p}, p.t, None)
    for k in also:
        assert torch.equal(also[k], got[k]), k


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad,shift", LAYOUTS)
def test_backward_matches_definition(rows, cols, pad, shift):
    for i, form in enumerate(FORMS):
        case = Case(rows, cols, pad, shift, form, seed=10 * i)
        if form[3]:
            check_backward(case)
            check_backward(case, use_dr=False)
        check_backward(case, use_dy=False)


@pytest.mark.parametrize("rows,cols", MANY)
def test_backward_of_many_rows(rows, cols):
    for i in (0, 1, 2):
        check_backward(Case(rows, cols, 0, 0, FORMS[i], seed=i))
    check_backward(Case(rows, cols, 8, 0, FORMS[3], seed=4))


def test_gradients_agree_with_differences():
    """d sum(y dy + r dr) against central differences of the definition in 64 bits, through a rounded forward pass of small values."""
    rows, cols, form = 3, 24, ("token", B.GATE_SILU, True, True)
    c = Case(rows, cols, 0, 0, form)
    dy, dr = normal(8, rows, cols), normal(9, rows, cols)

    def objective(x, o, gate, post, pre):
        n = o / torch.sqrt((o * o).mean(1, keepdim=True) + EPS) * post
        r = ALPHA * x + BETA * gate * torch.sigmoid(gate) * n
        return ((r / torch.sqrt((r * r).mean(1, keepdim=True) + EPS) * pre) * dy.double() + r * dr.double()).sum()
    leaves = [t.double() for t in (c.x.t, c.o.t, c.gate.t, c.post, c.pre)]
    r, y, rpost, rpre = (torch.empty(rows, cols, dtype=BF16, device="cuda") for _ in range(2)), None, vec(rows), vec(rows)
    r, y = r
    B.block_norm(c.x.t, c.o.t, r, y=y, rstd_post=rpost, rstd_pre=rpre, eps=EPS, **c.kw)
    out = [torch.empty_like(t) for t in (c.x.t, c.o.t, c.gate.t, c.post, c.pre)]
    ws = torch.empty(B.block_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda")
    B.block_norm_backward(dy, r, c.o.t, rpost, rpre, out[0], out[1], dr=dr, dgate=out[2], dpost_weight=out[3], dpre_weight=out[4], workspace=ws, **c.kw)
    for k, leaf in enumerate(leaves):
        grad, h = torch.zeros_like(leaf), 1e-5
        for i in range(leaf.numel()):
            step = torch.zeros_like(leaf).flatten()
            step[i] = h
            up, down = ([t + step.view_as(t) * s if j == k else t for j, t in enumerate(leaves)] for s in (1, -1))
            grad.flatten()[i] = (objective(*up) - objective(*down)) / (2 * h)
        # the backward pass reads r rounded to bfloat16: 2^-8 of each r, through a gradient whose slope in r / rms is a few units
        close(out[k], grad, 0.02 * grad.abs() + 0.03 * grad.abs().max(), str(k))


def test_rows_of_zeros_and_non_finite_values():
    rows, cols = 6, 512
    x, o = normal(1, rows, cols), normal(2, rows, cols)
    x[1], o[1] = 0, 0
    o[2, 5], x[3, 7] = INF, NAN
    gate = normal(3, 1, cols)
    gate[0, 9] = -INF                                    # a closed gate
    one = torch.ones(cols, dtype=BF16, device="cuda")
    r, y, y8, scale = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x, dtype=E4M3), vec(rows)
    B.block_norm(x, o, r, gate=gate, post_weight=one, pre_weight=one, y=y, y8=y8, y8_scale=scale, eps=EPS, activation=B.GATE_SIGMOID)
    assert (r[1] == 0).all() and (y[1] == 0).all() and (y8[1].float() == 0).all() and scale[1] == 0
    assert r[2, 5].isnan() and y[2].isnan().all()        # rstd 0, and infinity times 0
    assert y[3].isnan().all() and scale[3].isnan()
    for i in (0, 4, 5):
        assert r[i].isfinite().all() and torch.equal(r[i, 9], x[i, 9])
    silu = torch.empty_like(x)
    B.block_norm(x, o, silu, gate=gate, post_weight=one, eps=EPS, activation=B.GATE_SILU)
    assert silu[0].isfinite().all() and torch.equal(silu[0, 9], x[0, 9])
    d, dg = torch.empty_like(x), torch.empty_like(gate)
    ws = torch.empty(B.block_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda")
    for act in (B.GATE_SIGMOID, B.GATE_SILU):
        B.block_norm_backward(None, None, o[4:], (torch.ones(2, device="cuda")), None, None, d[4:], dr=x[4:], gate=gate, post_weight=one, dgate=dg, workspace=ws,
                              activation=act)
        assert d[4:].isfinite().all() and dg.isfinite().all() and dg[0, 9] == 0


@pytest.mark.parametrize("cols", [512, 515])
def test_rows_whose_squares_no_float_holds(cols):
    for size in (1e25, 3e38, 1e-25, 1e-37):
        o = (normal(1, 4, cols, dtype=F32).clamp(-1, 1) * size).to(BF16)
        x = torch.zeros_like(o)
        one = torch.ones(cols, dtype=BF16, device="cuda")
        r, y = torch.empty_like(o), torch.empty_like(o)
        B.block_norm(x, o, r, post_weight=one, pre_weight=one, y=y, eps=0.0)
        want = o.double() / torch.sqrt((o.double() ** 2).mean(1, keepdim=True))
        close(r, want, U * 1.01 * want.abs(), f"r {size}")
        B.block_norm(o, x, r, pre_weight=one, y=y, eps=0.0)
        close(y, want, U * 1.01 * want.abs(), f"y {size}")
        assert torch.equal(r, o)


def test_empty_extents():
    ws = torch.empty(B.block_norm_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    none = torch.empty(0, 64, dtype=BF16, device="cuda")
    one, dpost, dpre, dgate = torch.ones(64, dtype=BF16, device="cuda"), vec(64, BF16), vec(64, BF16), vec(64, BF16).view(1, 64)
    empty = torch.empty(0, device="cuda")
    B.block_norm(none, none, none, gate=one.view(1, 64), post_weight=one, pre_weight=one, y=none)
    B.block_norm_backward(none, none, none, empty, empty, none, none, gate=one.view(1, 64), post_weight=one, pre_weight=one, dgate=dgate, dpost_weight=dpost,
                          dpre_weight=dpre, workspace=ws)
    assert (dpost == 0).all() and (dpre == 0).all() and (dgate == 0).all()
    thin = torch.empty(3, 0, dtype=BF16, device="cuda")
    rpost, scale = vec(3) * 0, vec(3)
    B.block_norm(thin, thin, thin, post_weight=torch.empty(0, dtype=BF16, device="cuda"), rstd_post=rpost)
    assert rpost.isnan().all()
    B.block_norm(thin, thin, thin, pre_weight=torch.empty(0, dtype=BF16, device="cuda"), y8=torch.empty(3, 0, dtype=E4M3, device="cuda"), y8_scale=scale)
    assert (scale == 0).all()


def test_streams_graphs_and_repetition():
    rows, cols = 517, 2048
    c = Case(rows, cols, 0, 0, FORMS[0])
    dy, dr = normal(5, rows, cols), normal(6, rows, cols)

    def buffers():
        big = lambda: torch.empty(rows, cols, dtype=BF16, device="cuda")  # noqa: E731
        return dict(r=big(), y=big(), rpost=vec(rows), rpre=vec(rows), dx=big(), do=big(), dg=vec(cols, BF16).view(1, cols), dpost=vec(cols, BF16),
                    dpre=vec(cols, BF16), ws=torch.empty(B.block_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda"))

    def both(b, stream):
        B.block_norm(c.x.t, c.o.t, b["r"], y=b["y"], rstd_post=b["rpost"], rstd_pre=b["rpre"], eps=EPS, stream=stream, **c.kw)
        B.block_norm_backward(dy, b["r"], c.o.t, b["rpost"], b["rpre"], b["dx"], b["do"], dr=dr, dgate=b["dg"], dpost_weight=b["dpost"], dpre_weight=b["dpre"],
                              workspace=b["ws"], stream=stream, **c.kw)
    first = buffers()
    both(first, None)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [buffers() for _ in range(3)]
    for _ in range(5):
        for s, b in zip(streams, got):
            both(b, s)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        both(got[2], s)
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for b in got:
        for k in first:
            assert k == "ws" or torch.equal(b[k], first[k]), k


def test_offsets_beyond_32_bits():
    rows, cols, ld = 3, 512, (1 << 31) + 24
    raw = torch.empty(2 * ld + cols, dtype=BF16, device="cuda")
    o = raw.as_strided((rows, cols), (ld, 1))
    o.copy_(normal(1, rows, cols))
    x, one = normal(2, rows, cols), torch.ones(cols, dtype=BF16, device="cuda")
    far, near = torch.empty_like(x), torch.empty_like(x)
    B.block_norm(x, o, far, post_weight=one)
    B.block_norm(x, o.clone(), near, post_weight=one)
    assert torch.equal(far, near)
    B.block_norm_backward(None, None, x, torch.ones(rows, device="cuda"), None, None, o, dr=near, post_weight=one)
    B.block_norm_backward(None, None, x, torch.ones(rows, device="cuda"), None, None, far, dr=near, post_weight=one)
    assert torch.equal(o, far)
