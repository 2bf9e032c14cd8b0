"""The block norm's backward pass from x instead of the stored stream: gradients of r as it was before it was rounded.

Tolerances as in the tests of the block norm: U = 2^-8 for the one rounding of an output, `deep` for a float sum over a row, E = 2^-20 of the
magnitudes that go in for products, sums and gates.  r is formed anew within E of the magnitudes of its two terms; what that puts into
nr = r rstd_pre goes through the formulas below with the rest.
"""
import pytest
import torch

from ops_util import BF16, F32, U, Box, close, normal
from paper_2405_03637_b200 import binding as B
from test_gpu_block_norm import ALPHA, BETA, E, EPS, FORMS, LAYOUTS, Case, vec

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 7), (5, 64), (33, 257), (57, 104), (7, 768), (130, 1024), (19, 4096), (9, 5120), (3, 5632), (3, 8192), (2, 11008), (2, 20008), (2, 16001)]
MANY = [(6428, 96), (5000, 520), (13500, 136), (2400, 4096), (700, 5120), (460, 5632), (460, 8192), (700, 257)]


def check_from_x(c, use_dr=True, seed=60):
    rows, cols = c.rows, c.cols
    x64, o64 = c.x.t.double(), c.o.t.double()
    r, y, rpost, rpre = c.box(), c.box(), vec(rows) if c.post_on else None, vec(rows)
    B.block_norm(c.x.t, c.o.t, r.t, y=y.t, rstd_post=rpost, rstd_pre=rpre, eps=EPS, **c.kw)
    dy, dr = c.box(data=normal(seed, rows, cols)), c.box(data=normal(seed + 1, rows, cols))
    deep, rows_deep = (cols / 32 + 16) * 2.0 ** -23, (rows + 16) * 2.0 ** -23
    A = c.A if c.gate is not None else torch.ones(1, 1, dtype=torch.float64, device="cuda")
    w = c.post.double() if c.post_on else torch.ones(cols, dtype=torch.float64, device="cuda")
    rs_o = rpost.double()[:, None] if c.post_on else 1.0             # the forward call's, as the backward call takes them
    rs = rpre.double()[:, None]
    no = o64 * rs_o
    r64, r_off = ALPHA * x64 + BETA * A * no * w, E * ((ALPHA * x64).abs() + (BETA * A * no * w).abs())
    nr, nr_off = r64 * rs, rs * r_off
    q = dy.t.double() * c.pre.double()
    mean, spread = (q * nr).mean(1, keepdim=True), (q * nr).abs().mean(1, keepdim=True)
    mean_off = spread * deep + (q.abs() * nr_off).mean(1, keepdim=True)
    D = rs * (q - nr * mean) + (dr.t.double() if use_dr else 0)
    D_size = rs * (q.abs() + (nr * mean).abs()) + (dr.t.double().abs() if use_dr else 0)
    D_off = rs * (nr.abs() * mean_off + nr_off * mean.abs()) + E * D_size
    u, u_off = BETA * D, abs(BETA) * (D_off + E * D.abs())
    du, du_off = u * A, A.abs() * (u_off + E * u.abs())
    want, tol = {}, {}

    def expect(name, v, off):
        want[name], tol[name] = v, U * 1.001 * v.abs() + 1.02 * off + 1e-38
    expect("dpre_weight", (dy.t.double() * nr).sum(0), (rows_deep + E) * (dy.t.double() * nr).abs().sum(0) + (dy.t.double().abs() * nr_off).sum(0))
    expect("dx", ALPHA * D, ALPHA * (D_off + E * D.abs()))
    if c.post_on:
        h, h_off = du * w, w.abs() * (du_off + E * du.abs())
        m, s = (h * no).mean(1, keepdim=True), (h * no).abs().mean(1, keepdim=True)
        expect("dblock", rs_o * (h - no * m), rs_o * (h_off + E * h.abs() + no.abs() * ((h_off * no.abs()).mean(1, keepdim=True) + s * (deep + E))))
        expect("dpost_weight", (du * no).sum(0), ((du_off + E * du.abs()) * no.abs()).sum(0) + rows_deep * (du * no).abs().sum(0))
    else:
        expect("dblock", du, du_off)
    if c.gate is not None:
        un, un_off = u * no * w, (u_off + E * u.abs()) * (no * w).abs()
        if c.gate.rows == 1 and rows > 1:
            s, s_off = un.sum(0, keepdim=True), un_off.sum(0, keepdim=True) + rows_deep * un.abs().sum(0, keepdim=True)
            expect("dgate", s * c.slope, s_off * c.slope_mag + 2 * E * s.abs() * c.slope_mag)
        else:
            expect("dgate", un * c.slope, un_off * c.slope_mag + 2 * E * un.abs() * c.slope_mag)
    ws = torch.full((B.block_norm_workspace_bytes(cols),), 0xFF, dtype=torch.uint8, device="cuda")

    def outputs(names):
        return {k: vec(cols, BF16) if k in ("dpost_weight", "dpre_weight") else c.box(n=c.gate.rows if k == "dgate" else rows) for k in names}

    def call(out, dy_t=dy.t, dr_t=dr.t):
        t = {k: v.t if isinstance(v, Box) else v for k, v in out.items()}
        got = dict(t)
        B.block_norm_backward(dy_t, None, c.o.t, rpost, rpre, t.pop("dx", None), t.pop("dblock", None), dr=dr_t if use_dr else None, workspace=ws, x=c.x.t, **c.kw, **t)
        return got
    whole = outputs(want)
    got = call(whole)
    for k in want:
        close(got[k], want[k], tol[k], k)
        assert not isinstance(whole[k], Box) or whole[k].untouched_outside()
    for k in want:                                       # one output at a time gives the same bits
        assert torch.equal(call(outputs([k]))[k], got[k]), k
    place = {k: v for k, v in outputs(want).items() if k not in ("dx", "dblock")}
    p, d = c.box(data=dy.t), c.box(data=dr.t)            # in the place of the gradients that came in
    also = call({**place, "dx": d, "dblock": p}, p.t, d.t) if use_dr else call({**place, "dblock": p}, p.t, None)
    for k in also:
        assert torch.equal(also[k], got[k]), k


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad,shift", LAYOUTS)
def test_from_x_matches_definition(rows, cols, pad, shift):
    for i, form in enumerate(FORMS):
        if form[3]:
            case = Case(rows, cols, pad, shift, form, seed=10 * i)
            check_from_x(case, use_dr=True)
            check_from_x(case, use_dr=False)


@pytest.mark.parametrize("rows,cols", MANY)
def test_from_x_of_many_rows(rows, cols):
    for i in (0, 1, 2):
        check_from_x(Case(rows, cols, 0, 0, FORMS[i], seed=i))


@pytest.mark.parametrize("rows,cols", [(57, 104), (6428, 96), (57, 103)])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_weight_gradient_where_one_column_holds_most_of_a_row(rows, cols, gate):
    """dpre_weight against the whole definition in 64 bits, forward pass included: one rounding of the result, and of each term of the sum (one dy nr
    for each row) the roundings in float of r (E of its magnitudes), of 1 / rms (`deep`) and of the sum.  (A stream stored in bfloat16 would put 2^-8 of
    each term in.)"""
    g = torch.Generator(device="cuda").manual_seed(2)
    big = torch.rand(cols, generator=g, device="cuda") < 1 / 64
    big[cols // 2] = True
    x = (normal(3, rows, cols, dtype=F32) * torch.where(big, 24.0, 1.0)).to(BF16)
    o, dy = normal(4, rows, cols, std=0.5), normal(5, rows, cols, std=1e-3)
    post, pre = (1 + 0.2 * normal(6, 2, cols, dtype=F32)).to(BF16)
    t = None if gate == "none" else normal(7, 1 if gate == "channel" else rows, cols)
    kw = dict(gate=t, post_weight=post, pre_weight=pre, residual_scale=0.9, block_scale=0.3)
    r, y, rpost, rpre, dpre = torch.empty_like(x), torch.empty_like(x), vec(rows), vec(rows), vec(cols, BF16)
    ws = torch.empty(B.block_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda")
    B.block_norm(x, o, r, y=y, rstd_post=rpost, rstd_pre=rpre, eps=EPS, **kw)
    B.block_norm_backward(dy, None, o, rpost, rpre, None, None, dpre_weight=dpre, workspace=ws, x=x, **kw)
    n = o.double() / torch.sqrt((o.double() ** 2).mean(1, keepdim=True) + EPS) * post.double() * (1.0 if t is None else t.double())
    r64, size = 0.9 * x.double() + 0.3 * n, 0.9 * x.double().abs() + 0.3 * n.abs()
    rms = torch.sqrt((r64 * r64).mean(1, keepdim=True) + EPS)
    want = (dy.double() * r64 / rms).sum(0)
    deep = (cols / 32 + 16) * 2.0 ** -23
    terms = (dy.double().abs() * size / rms).sum(0)
    close(dpre, want, U * 1.001 * want.abs() + (2 * deep + 2 * E + (rows + 16) * 2.0 ** -23) * terms, "dpre_weight")


def test_streams_and_graphs():
    rows, cols = 517, 2048
    c = Case(rows, cols, 0, 0, FORMS[0])
    dy, dr = normal(5, rows, cols), normal(6, rows, cols)

    def buffers():
        big = lambda: torch.empty(rows, cols, dtype=BF16, device="cuda")  # noqa: E731
        return dict(r=big(), y=big(), rpost=vec(rows), rpre=vec(rows), dx=big(), do=big(), dg=vec(cols, BF16).view(1, cols), dpost=vec(cols, BF16),
                    dpre=vec(cols, BF16), ws=torch.empty(B.block_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda"))

    def both(b, stream):
        B.block_norm(c.x.t, c.o.t, b["r"], y=b["y"], rstd_post=b["rpost"], rstd_pre=b["rpre"], eps=EPS, stream=stream, **c.kw)
        B.block_norm_backward(dy, None, c.o.t, b["rpost"], b["rpre"], b["dx"], b["do"], dr=dr, dgate=b["dg"], dpost_weight=b["dpost"], dpre_weight=b["dpre"],
                              workspace=b["ws"], stream=stream, x=c.x.t, **c.kw)
    first, streams, got = buffers(), [torch.cuda.Stream() for _ in range(2)], [buffers() for _ in range(3)]
    both(first, None)
    torch.cuda.synchronize()
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
    x = raw.as_strided((rows, cols), (ld, 1))
    x.copy_(normal(1, rows, cols))
    o, dy, one = normal(2, rows, cols), normal(3, rows, cols), torch.ones(cols, dtype=BF16, device="cuda")
    rpre, far, near = torch.full((rows,), 0.7, device="cuda"), torch.empty_like(o), torch.empty_like(o)
    for from_x, to in ((x, far), (x.clone(), near)):
        B.block_norm_backward(dy, None, o, None, rpre, to, None, pre_weight=one, x=from_x)
    assert torch.equal(far, near)


@pytest.mark.parametrize("cols", [200, 512, 515, 4096, 5632, 16001])
@pytest.mark.parametrize("act", [B.GATE_SIGMOID, B.GATE_SILU])
@pytest.mark.parametrize("token", [False, True])
def test_closed_gates_rows_of_zeros_and_values_that_are_no_numbers(cols, act, token):
    """A gate of minus infinity lets nothing through, either way; a row's NaN stays in its row (and in the sums over rows)."""
    rows = 7
    x, o, dy = normal(1, rows, cols), normal(2, rows, cols), normal(3, rows, cols)
    gate = normal(4, rows if token else 1, cols)
    gate[:, 9], gate[:, 11] = float("-inf"), -3e38
    x[2], o[2] = 0, 0
    one = torch.ones(cols, dtype=BF16, device="cuda")
    ws = torch.empty(B.block_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda")
    kw = dict(gate=gate, post_weight=one, pre_weight=one, activation=act)
    for bad in (None, 5):
        if bad is not None:
            dy[bad, 1] = float("nan")
        r, y, rpost, rpre = torch.empty_like(x), torch.empty_like(x), vec(rows), vec(rows)
        B.block_norm(x, o, r, y=y, rstd_post=rpost, rstd_pre=rpre, eps=EPS, **kw)
        dx, do, dg, dpost, dpre = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gate), vec(cols, BF16), vec(cols, BF16)
        B.block_norm_backward(dy, None, o, rpost, rpre, dx, do, dgate=dg, dpost_weight=dpost, dpre_weight=dpre, workspace=ws, x=x, **kw)
        whole = [i for i in range(rows) if i != bad]
        assert dx[whole].isfinite().all() and do[whole].isfinite().all()
        if bad is None:
            assert dpost.isfinite().all() and dpre.isfinite().all() and dg.isfinite().all() and (dg[:, 9] == 0).all() and (dpost[[9, 11]] == 0).all()
        else:
            assert dx[bad].isnan().all() and do[bad].isnan().all() and dpre[1].isnan()
