"""Training-step operators at the edges of their variants: sizes at which a launch changes its kind, several turns of
persistent kernels, zeros with a sign, values at the ends of the range."""
import subprocess
import sys
from pathlib import Path

import pytest
import torch

import test_gpu_training_ops as ops
from ops_util import BF16, E4M3, U, close, normal
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

# Rows whose slice takes between 43 and 49 KB of shared memory, each kernel's first launch of the process: the kernel's own
# 4.5 KB come on top of it, and beyond 48 KB in all a launch needs leave that an earlier, larger launch may have asked for.
FIRST_LAUNCHES = """
import torch
from paper_2405_03637_b200 import binding as B
for dtype, vocab in ((torch.bfloat16, 24_000), (torch.float32, 12_000)):
    rows, k = 300, 16
    z = torch.randn(rows, vocab, device="cuda").to(dtype)
    at, top = torch.arange(k, device="cuda").repeat(rows, 1), torch.zeros(rows, k, device="cuda")
    loss, dz = torch.empty(rows, device="cuda"), torch.empty_like(z)
    B.distill_loss_and_grad(z, at, top, 1.0, torch.ones(rows, device="cuda"), loss, dz)
    want = torch.logsumexp(z.double(), 1) - z[:, :k].double().mean(1) - torch.log(torch.tensor(float(k)))
    assert (loss.double() - want).abs().max() < 1e-4, vocab
"""


def test_first_launches_of_every_size_of_shared_memory():
    p = subprocess.run([sys.executable, "-c", FIRST_LAUNCHES], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-2000:]


@pytest.mark.parametrize("cols", [300, 304, 4096])
def test_rounding_to_8_bits_keeps_the_sign_of_zero(cols):
    # every code of the format, both zeros among them, in rows that go by elements and by vectors: the scale is 1
    codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    codes = codes[~codes.view(E4M3).float().isnan()]
    x = torch.zeros(3, cols, dtype=BF16, device="cuda")
    x[:, :codes.numel()] = codes.view(E4M3).float().to(BF16)
    x[1] *= 0.37
    x[2, codes.numel():] = -0.0
    x[2, :codes.numel()] = normal(1, codes.numel(), std=1e-38)       # beyond the divisors of the shortcut
    q, scale = torch.empty_like(x, dtype=E4M3), torch.empty(3, device="cuda")
    B.quantize_rows(x, q, scale)
    assert scale[0] == 1 and torch.equal(q[0, :codes.numel()].view(torch.uint8), codes)
    want = (x.float() / scale[:, None]).to(E4M3)
    assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("rows,cols", [(6, 257), (6, 1000), (6, 4096), (6, 16384), (6, 33_000), (600, 256), (600, 1024)])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_norm_of_rows_whose_squares_no_float_holds(rows, cols, eps):
    x, dy, weight = normal(1, rows, cols), normal(2, rows, cols), normal(3, cols)
    for i, size in enumerate((1e20, -3e37, 1e-25, 1e-12)):
        x[i::6] *= size
    x[4::6] = torch.finfo(BF16).max
    new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    y, y8, scale, rstd = torch.empty_like(x), torch.empty_like(x, dtype=E4M3), new(rows), new(rows)
    B.add_rms_norm(x, None, weight, eps, y=y, y8=y8, y8_scale=scale, rstd=rstd)
    r, w = x.double(), weight.double()
    rstd64 = 1 / torch.sqrt((r * r).mean(1) + eps)
    y64 = r * rstd64[:, None] * w
    # the sum of squares as for ordinary rows; 1 / 3e38 is a subnormal float of 22 bits
    deep = (cols / 32 + 16) * 2.0 ** -23 + 2.0 ** -22
    close(rstd, rstd64, deep * rstd64, "rstd")
    close(y, y64, (U * 1.001 + 2 * deep) * y64.abs() + 2.0 ** -133, "y")       # (half of bfloat16's smallest step is 2^-134)
    scale64 = y64.abs().amax(1) / 448
    close(scale, scale64, (2 * deep + 2.0 ** -22) * scale64, "scale")
    close(y8.double() * scale.double()[:, None], y64, y64.abs() * (2.0 ** -4 + 4 * deep) + scale64[:, None] * 2.0 ** -10 * 1.001, "y8")
    dx, dweight = torch.empty_like(x), new(cols, dtype=BF16)
    B.add_rms_norm_backward(dy, x, rstd, weight, dx, dweight, torch.empty(B.rms_norm_workspace_bytes(cols), dtype=torch.uint8, device="cuda"))
    n, g = r * rstd.double()[:, None], dy.double() * w
    want = (g - n * (g * n).mean(1, keepdim=True)) * rstd.double()[:, None]
    terms = rstd.double()[:, None] * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    close(dx, want, U * 1.001 * want.abs() + (deep + 2.0 ** -20) * terms + 2.0 ** -133, "dx")
    dw64, mag = (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)
    close(dweight, dw64, U * 1.001 * dw64.abs() + (rows + 8) * 2.0 ** -23 * mag, "dweight")


def test_norm_of_rows_without_columns_writes_what_it_promises():
    x, w = torch.empty(3, 0, dtype=BF16, device="cuda"), torch.empty(0, dtype=BF16, device="cuda")
    rstd, scale = torch.full((3,), 7.0, device="cuda"), torch.full((3,), 7.0, device="cuda")
    B.add_rms_norm(x, None, w, 1e-5, y=torch.empty_like(x), y8=torch.empty_like(x, dtype=E4M3), y8_scale=scale, rstd=rstd)
    assert rstd.isnan().all() and (scale == 0).all()         # the mean of nothing, and the largest of nothing


def test_temperatures_whose_reciprocal_is_too_large_are_refused():
    z, at, top, loss = normal(1, 2, 64), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, device="cuda"), torch.zeros(2, device="cuda")
    for tau in (3.2e-39, 4.2e-39):                           # 1 / t is a float, 1 / (t ln 2) is not
        with pytest.raises(B.CollageError) as e:
            B.distill_loss(z, at, top, tau, loss)
        assert e.value.status == B.ERR_ARG
    B.distill_loss(z, at, top, 4.4e-39, loss)
    assert not loss.isnan().any()


def test_three_dimensions_without_columns():
    # [2, 3, 0] is six rows of nothing, as [6, 0] is
    x, q, scale = torch.empty(2, 3, 0, dtype=BF16, device="cuda"), torch.empty(2, 3, 0, dtype=E4M3, device="cuda"), torch.full((6,), 7.0, device="cuda")
    B.quantize_rows(x, q, scale)
    assert (scale == 0).all()
    h = torch.full((2, 3, 8), 7.0, dtype=BF16, device="cuda")
    none = torch.empty(8, 0, dtype=BF16, device="cuda")
    B.gated_ffn(x, none, none, h)
    assert (h == 0).all()


def test_the_operators_want_their_stream_named_beside_the_default_one():
    x, q, scale = normal(1, 4, 64), torch.zeros(4, 64, dtype=E4M3, device="cuda"), torch.zeros(4, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with pytest.raises(B.CollageError) as e:
            B.quantize_rows(x, q, scale)
        assert e.value.status == B.ERR_ARG and "stream" in str(e.value)
        B.quantize_rows(x, q, scale, stream=torch.cuda.current_stream())
    side.synchronize()
    assert (scale > 0).all()
    with torch.cuda.stream(side):
        B.quantize_rows(x, q, scale, stream=torch.cuda.default_stream())
    torch.cuda.synchronize()


# ------------------------------------------------------------------- several turns of the kernels that walk over their work ---

@pytest.mark.parametrize("rows,cols", [(25_000, 64), (6000, 1000), (1700, 4096), (750, 12_288), (750, 16_384)])
def test_norm_backward_over_five_rows_a_group(rows, cols):
    ops.test_norm_backward_matches_definition(rows, cols, 0, 0)


@pytest.mark.parametrize("rows,vocab,dtype", [(700, 32_000, torch.float32), (700, 70_001, BF16), (80, 400_003, BF16)])
def test_distillation_over_several_rows_a_cluster(rows, vocab, dtype):
    z = normal(5, rows, vocab, std=2.0, dtype=dtype)
    at, top = ops.teacher(6, rows, vocab, 24)
    at[2::7] = -1                                            # rows without entries, and rows that weigh nothing, between others
    weight = torch.linspace(0.5, 1.5, rows, device="cuda")
    weight[::5] = 0
    ops.check_distill(z, at, top, 2.0, weight)


# 74 pairs of blocks: tiles for more than three turns, in the forward pass, in dx or in the weight gradients, with few and many
# blocks of K, and more than eight rows of tiles with an incomplete last group
@pytest.mark.parametrize("tokens,width,ffn", [(4900, 136, 2056), (4095, 1032, 2056), (4095, 4104, 264), (1300, 2056, 4104)])
def test_feed_forward_over_several_tiles_a_pair(tokens, width, ffn):
    ops.test_gated_forward_and_backward_match_definition(tokens, width, ffn, 0, 0, B.ACT_SILU)


@pytest.mark.parametrize("tokens,width,ffn", [(4900, 144, 2064), (4095, 1040, 2064)])
def test_feed_forward_in_8_bits_over_several_tiles_a_pair(tokens, width, ffn):
    ops.test_gated_8_bits_matches_definition(tokens, width, ffn, 0, 0)


def test_many_tiles_give_the_same_bits_again():
    launch, o = ops.one_of_each(tokens=4900, width=1032, ffn=2056, vocab=4099)
    launch()
    first = ops.bits_of(o)
    for _ in range(3):
        for v in o.values():
            v.view(torch.uint8).zero_()
        launch()
        now = ops.bits_of(o)
        assert all(torch.equal(first[k], now[k]) for k in first) and B.pipeline_fault() == 0
