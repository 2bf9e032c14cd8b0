"""Token log-probabilities, the clipped policy loss and the preference loss against their definitions in 64 bits.

Tolerances.  Exponentials are within 2^-21 (2 units of a float's last place, and the rounding of an argument x adds |x| 2^-23); a row's
sum, whose terms a thread adds up by two chains, is within (vocab / 512 + 40) 2^-23 of itself; `REL` has both.  A log-probability is
that sum's relative error off, plus a float's rounding of the difference to the maximum and of the result.  Results are rounded once:
half a unit in the last place, U (bfloat16) or 2^-24 (float) of the value.
"""
import math

import pytest
import torch

from ops_util import BF16, F32, U, Box, close, normal
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
ROUND = {BF16: U, F32: 2.0 ** -24}
TINY = 2.0 ** -125                          # exponentials below a float's normal range are zeros


def rel_of(vocab):
    return (vocab / 512 + 40) * 2.0 ** -23 + 2.0 ** -21


def vec(n, dtype=F32):
    return torch.full((n,), NAN, dtype=dtype, device="cuda")


# (rows, vocab, row stride beyond the columns, elements off a 16-byte boundary)
SHAPES = [(1, 1, 0, 0), (3, 2, 0, 0), (2, 9, 0, 1), (5, 100, 0, 0), (4, 1000, 3, 1), (7, 4097, 0, 0), (3, 8192, 8, 0), (2, 8191, 0, 3), (1, 32000, 0, 0),
          (6, 50257, 0, 0), (2, 131072, 0, 0), (1, 131071, 5, 1), (301, 1003, 0, 0), (700, 512, 0, 0), (1200, 257, 1, 0), (160, 32000, 0, 0), (149, 50257, 0, 0),
          (3, 300_001, 0, 0), (2, 1_000_003, 0, 1)]


class Rows:
    """Logits with a few peaks, targets of which some are absent, and the definition's values in 64 bits."""

    def __init__(self, rows, vocab, pad, shift, dtype, tau, index=torch.int64, seed=0, offset=0.0):
        self.rows, self.vocab, self.tau, self.dtype = rows, vocab, tau, dtype
        self.box = lambda data=None: Box(rows, vocab, dtype, vocab + pad, shift, data)
        g = torch.Generator(device="cuda").manual_seed(seed)
        z = torch.randn((rows, vocab), generator=g, device="cuda") * 3 + offset
        z[torch.arange(rows, device="cuda"), torch.randint(0, vocab, (rows,), generator=g, device="cuda")] += 9
        self.z = self.box(z.to(dtype))
        y = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        y[::2] = self.z.t[::2].float().argmax(1)
        y[0], y[-1] = 0, vocab - 1
        if rows > 4:
            y[1], y[3] = -1, vocab                      # no targets
        self.y = y.to(index)
        self.counts = (y >= 0) & (y < vocab)
        self.safe = torch.where(self.counts, y, 0)
        z64 = self.z.t.double() / tau
        self.lse = torch.logsumexp(z64, 1)
        at = z64.gather(1, self.safe[:, None])[:, 0]
        self.logp = torch.where(self.counts, at - self.lse, 0.0)
        self.top, self.at = z64.amax(1), at
        self.logp_off = rel_of(vocab) + 2.0 ** -23 * ((self.top - at).abs() + self.logp.abs()) + 2.0 ** -23

    def gradient(self, coef, coef_off):
        """d logits and their tolerance for gradients `coef` of logp that are `coef_off` off."""
        z64 = self.z.t.double() / self.tau
        q = (z64 - self.lse[:, None]).exp()
        gain, off = (coef / self.tau)[:, None], (coef_off / self.tau)[:, None]
        hot = torch.zeros_like(q).scatter_(1, self.safe[:, None], 1.0)
        want = torch.where(self.counts[:, None], gain * (hot - q), 0.0)
        rel = rel_of(self.vocab) + 2.0 ** -22 * ((self.top[:, None] - z64).abs() + 2)
        size = (hot + q) * 1.001
        return want, ROUND[self.dtype] * want.abs() * 1.001 + gain.abs() * (q * rel + hot * 2.0 ** -22) + off * size + (gain.abs() + 1) * TINY


def forms(seed):
    return [(BF16, 1.0, torch.int64), (F32, 0.7, torch.int32)] if seed % 2 == 0 else [(F32, 1.0, torch.int64), (BF16, 2.5, torch.int32)]


@pytest.mark.parametrize("rows,vocab,pad,shift", SHAPES)
def test_logp_and_its_backward_match_definition(rows, vocab, pad, shift):
    for dtype, tau, index in forms(rows):
        r = Rows(rows, vocab, pad, shift, dtype, tau, index)
        logp, stats, bare, rest = vec(rows), vec(2 * rows).view(rows, 2), vec(rows), vec(rows)
        B.token_logp(r.z.t, r.y, tau, logp, stats=stats, logp_rest=rest)
        assert (rest.abs() <= 2.0 ** -24 * logp.abs()).all()         # half a unit of logp's last place at most
        # both together: the row's sum is within rel_of(vocab), the rest is in 64 bits but for the difference to the maximum in float
        close(logp.double() + rest.double(), r.logp, torch.where(r.counts, rel_of(vocab) + 2.0 ** -24 * (r.top - r.at).abs(), 0.0), "logp and rest")
        B.token_logp(r.z.t, r.y, tau, bare)
        assert torch.equal(logp, bare)
        close(logp, r.logp, torch.where(r.counts, r.logp_off, 0.0), "logp")
        close(stats[:, 0], torch.where(r.counts, r.z.t.float().amax(1), 0.0), 0.0, "maximum")
        close(stats[:, 1], torch.where(r.counts, (r.lse - r.top).exp(), 0.0), rel_of(vocab) * (r.lse - r.top).exp(), "sum")
        grad = normal(5, rows, dtype=F32)
        if rows > 2:
            grad[2] = 0
        for d in (r.box(), r.z):                        # and in the logits' place
            want, tol = r.gradient(grad.double(), 0 * grad.double())
            B.token_logp_backward(r.z.t, r.y, tau, stats, grad, d.t)
            close(d.t, want, tol, "dlogits")
            assert d.untouched_outside()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [0.7, 1.0, 1.3])
def test_errors_of_logp_do_not_add_up(tau, dtype):
    """A sequence sums thousands of log-probabilities: their mean is off by less than a rounding of the sum of exponentials, 2^-23 (an
    exponential is off by up to 2^-22, both ways, and log2(e) / tau in one float by up to 2^-23, which a difference of 8 in the logits
    would make 2^-20; the 512 rows' own spread adds 2^-22 / sqrt(512))."""
    rows, vocab = 512, 13304
    g = torch.Generator(device="cuda").manual_seed(17)
    z = (torch.randn((rows, vocab), generator=g, device="cuda") * 2).to(dtype)
    y = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    want = (z.double() / tau).gather(1, y[:, None])[:, 0] - torch.logsumexp(z.double() / tau, 1)
    logp, rest = vec(rows), vec(rows)
    B.token_logp(z, y, tau, logp, logp_rest=rest)
    assert (logp.double() + rest.double() - want).mean().abs() < 2.0 ** -23


def policy_inputs(r, seed=3):
    """Ratios on both sides of each bound, none within a hundredth of one; advantages of both signs and zero."""
    pick = torch.arange(r.rows, device="cuda")
    d = torch.tensor([0.0, -0.5, 0.1, 0.5, -0.1, 1.5, -2.0], device="cuda", dtype=torch.float64)[pick % 7]
    k = torch.tensor([0.0, 0.3, -0.4, 0.01, 2.0], device="cuda", dtype=torch.float64)[pick % 5]
    adv = torch.tensor([1.0, -0.7, 0.0, 2.5], device="cuda")[pick % 4] * (1 + 0.1 * torch.rand(r.rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
    weight = torch.tensor([0.5, 1.0, 0.25], device="cuda")[pick % 3].clone()
    if r.rows > 6:
        weight[5] = 0
    return (r.logp - d).float(), (r.logp + k).float(), adv, weight


def policy64(r, old, ref, adv, weight, low, high, klw):
    live = r.counts & (weight != 0)
    a = adv.double()
    ratio = torch.ones_like(r.logp) if old is None else (r.logp - old.double()).exp()
    ratio_off = 0 * ratio if old is None else ratio * (r.logp_off + 2.0 ** -22 * ((r.logp - old.double()).abs() + 2))
    free, held = ratio * a, ratio.clamp(1 - low, 1 + high) * a
    clipped = held < free
    loss, coef, coef_off = -torch.where(clipped, held, free), torch.where(clipped, 0.0, -free), torch.where(clipped, 0.0, ratio_off * a.abs())
    loss_off = torch.where(clipped, 0.0, ratio_off * a.abs()) + 2.0 ** -22 * loss.abs()
    kl, kl_off = torch.zeros_like(ratio), torch.zeros_like(ratio)
    if ref is not None:
        k = ref.double() - r.logp
        kl = torch.special.expm1(k) - k
        kl_off = torch.special.expm1(k).abs() * r.logp_off + r.logp_off ** 2 + 2.0 ** -23 * kl
        loss, loss_off = loss + klw * kl, loss_off + klw * kl_off + 2.0 ** -22 * klw * kl
        coef, coef_off = coef - klw * torch.special.expm1(k), coef_off + klw * (k.exp() * r.logp_off + 2.0 ** -22 * torch.special.expm1(k).abs())
    w = torch.where(live, weight.double(), 0.0)
    coef_off = w * (coef_off + 2.0 ** -22 * coef.abs())
    zero = lambda t: torch.where(live, t, 0.0)  # noqa: E731
    return live, w * loss, w * (loss_off + 2.0 ** -22 * loss.abs()), zero(kl), zero(kl_off), w * coef, coef_off


@pytest.mark.parametrize("rows,vocab,pad,shift", SHAPES)
def test_policy_matches_definition(rows, vocab, pad, shift):
    for dtype, tau, index in forms(rows):
        r = Rows(rows, vocab, pad, shift, dtype, tau, index, seed=1)
        old, ref, adv, weight = policy_inputs(r)
        for with_old, with_ref in ((True, True), (True, False), (False, True)):
            o, f, klw = old if with_old else None, ref if with_ref else None, 0.2 if with_ref else 0.0
            live, loss64, loss_off, kl64, kl_off, coef, coef_off = policy64(r, o, f, adv, weight, 0.2, 0.3, klw)
            want, tol = r.gradient(coef, coef_off)
            loss, logp, kl, d = vec(rows), vec(rows), vec(rows) if with_ref else None, r.box()
            kw = dict(old_logp=o, ref_logp=f, clip_low=0.2, clip_high=0.3, kl_weight=klw)
            B.policy_loss_and_grad(r.z.t, r.y, tau, adv, weight, loss, d.t, logp=logp, kl=kl, **kw)
            close(logp, torch.where(live, r.logp, 0.0), r.logp_off, "logp")
            close(loss, loss64, loss_off + 1e-38, "loss")
            if with_ref:
                close(kl, kl64, kl_off + 1e-38, "kl")
            close(d.t, want, tol, "dlogits")
            assert d.untouched_outside()
            assert (loss[~live] == 0).all() and (logp[~live] == 0).all() and (d.t[~live] == 0).all()
            # the same bits without the optional outputs, and in the logits' place
            only, place = vec(rows), r.box(r.z.t)
            B.policy_loss_and_grad(place.t, r.y, tau, adv, weight, only, place.t, **kw)
            assert torch.equal(only, loss) and torch.equal(place.t, d.t) and place.untouched_outside()


def test_policy_gradient_agrees_with_differences():
    rows, vocab, tau = 6, 37, 0.8
    r = Rows(rows, vocab, 0, 0, F32, tau)
    old, ref, adv, weight = policy_inputs(r)

    def objective(z):
        logp = z.div(tau).log_softmax(1).gather(1, r.safe[:, None])[:, 0]
        ratio = (logp - old.double()).exp()
        k = ref.double() - logp
        each = -torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv) + 0.3 * (k.exp() - k - 1)
        return (torch.where(r.counts, each, 0.0) * weight).sum()
    z, h, grad = r.z.t.double(), 1e-5, torch.zeros(rows, vocab, dtype=torch.float64, device="cuda")
    for i in range(rows):
        for j in range(vocab):
            e = torch.zeros_like(z)
            e[i, j] = h
            grad[i, j] = (objective(z + e) - objective(z - e)) / (2 * h)
    d, loss = torch.empty_like(r.z.t), vec(rows)
    B.policy_loss_and_grad(r.z.t, r.y, tau, adv, weight, loss, d, old_logp=old, ref_logp=ref, kl_weight=0.3)
    close(d, grad, 1e-5 * (1 + grad.abs()), "against differences")          # h^2, and 1e-13 / h of rounding
    assert abs(float(loss.double().sum()) - float(objective(z))) < 1e-5


def test_policy_bounds_and_extreme_ratios():
    z = torch.zeros(8, 4, device="cuda")                                     # logp = -log 4 everywhere
    y = torch.zeros(8, dtype=torch.int32, device="cuda")
    base = -math.log(4)
    old = torch.tensor([base, base - 200, base - 200, base + 200, base + 200, base - 200, base, -INF], device="cuda")
    adv = torch.tensor([0.0, 1.0, 0.0, 1.0, -1.0, -1.0, 3.0, 0.0], device="cuda")
    one, loss, d = torch.ones(8, device="cuda"), vec(8), torch.empty_like(z)
    B.policy_loss_and_grad(z, y, 1.0, adv, one, loss, d, old_logp=old, clip_low=0.5, clip_high=1.0)
    # a ratio of infinity: bounded for A > 0, nothing for A = 0, infinite for A < 0
    assert loss.tolist()[:5] == [0.0, -2.0, 0.0, 0.0, 0.5] and loss[5] == INF and loss[7] == 0
    close(loss[6:7], torch.tensor([-3.0], device="cuda"), 2e-6, "ratio 1")
    assert (d[[0, 1, 2, 4, 7]] == 0).all() and (d[3] == 0).all()
    close(d[6], torch.tensor([-2.25, 0.75, 0.75, 0.75], device="cuda"), 2e-6, "gradient")
    B.policy_loss_and_grad(z, y, 1.0, adv, one, loss, d, old_logp=old, clip_low=1.0, clip_high=INF)      # no bounds
    assert loss[1] == -INF and loss[2] == 0
    # a KL term of infinity is left out at weight 0
    ref, kl = torch.full((8,), 1000.0, device="cuda"), vec(8)
    B.policy_loss_and_grad(z, y, 1.0, adv, one, loss, d, ref_logp=ref, kl_weight=0.0, kl=kl)
    assert (kl == INF).all() and loss.isfinite().all() and d.isfinite().all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [600, 50257])
def test_non_finite_and_far_logits(vocab, dtype):
    low = torch.finfo(dtype).min
    z = normal(1, 12, vocab).to(dtype)
    y = torch.full((12,), 5, device="cuda")
    z[0] = low                                            # uniform
    z[1] = -INF                                           # no distribution
    z[2, 7], z[3, 7] = NAN, INF
    z[4, 100:] = -INF                                     # most of the vocabulary ruled out
    z[5, 5] = -INF                                        # the target ruled out
    z[6] = z[6] * 1e3 + 3e4
    z[7], z[7, 5] = low, -low                             # the whole range
    z[8] = NAN                                            # not read: no target
    y[8] = -1
    z[9] = INF                                            # not read: no weight
    z[10, :] = -3e38
    z[10, 5] = 0
    weight = torch.ones(12, device="cuda")
    weight[9] = 0
    logp, stats, loss, d, back = vec(12), vec(24).view(12, 2), vec(12), torch.empty_like(z), torch.empty_like(z)
    B.token_logp(z, y, 1.0, logp, stats=stats)
    adv = torch.ones(12, device="cuda")
    B.policy_loss_and_grad(z, y, 1.0, adv, weight, loss, d)
    B.token_logp_backward(z, y, 1.0, stats, torch.ones(12, device="cuda"), back)
    close(logp[0], torch.tensor(-math.log(vocab), device="cuda"), 1e-5, "uniform")
    q = torch.full((vocab,), 1 / vocab, dtype=torch.float64, device="cuda")
    q[5] -= 1
    close(back[0], -q, (ROUND[dtype] + 1e-5) * q.abs(), "uniform gradient")
    for i in (1, 2, 3):
        assert logp[i].isnan() and back[i].isnan().all() and d[i].isnan().all(), i
    want = torch.log_softmax(z[4, :100].double(), 0)[5]
    close(logp[4], want, 1e-5, "ruled out")
    assert (back[4, 100:] == 0).all() and logp[5] == -INF and back[5].isfinite().all() and back[5, 5] == 1
    close(logp[6], torch.log_softmax(z[6].double(), 0)[5], 1e-3 + 2.0 ** -20 * 3e4, "far from zero")
    assert logp[7] == 0 and (back[7] == 0).all() and logp[10] == 0
    for t in (d, back):
        assert (t[8] == 0).all()
    assert logp[8] == 0 and loss[8] == 0 and (stats[8] == 0).all() and loss[9] == 0 and (d[9] == 0).all()


def sequences(lengths, gap=0, tail=0):
    o, at = [], gap
    for n in lengths:
        o.append(at)
        at += n
    return o + [at], at + tail


@pytest.mark.parametrize("lengths,gap,tail", [([3, 2], 0, 0), ([1, 0], 0, 0), ([0, 0], 2, 3), ([5, 700, 1300, 1], 4, 9), ([2000, 4096, 17, 0, 0, 33], 0, 1),
                                              ([7] * 300, 1, 1)])
@pytest.mark.parametrize("average", [False, True])
def test_preference_matches_definition(lengths, gap, tail, average):
    o, rows = sequences(lengths, gap, tail)
    pairs, vocab = len(lengths) // 2, 50
    logp, ref = -normal(1, rows, dtype=F32).abs() * 4, -normal(2, rows, dtype=F32).abs() * 4
    g = torch.Generator(device="cuda").manual_seed(3)
    y = torch.randint(-9, vocab + 9, (rows,), generator=g, device="cuda")
    counts = ((y >= 0) & (y < vocab)).cpu()
    w = torch.rand(pairs, generator=g, device="cuda")
    for index, offset_type, use_ref, use_w, smooth, margin in ((torch.int32, torch.int64, True, True, 0.1, 0.2), (torch.int64, torch.int32, False, False, 0.0, 0.0),
                                                               (torch.int64, torch.int32, True, False, 1.0, -0.5)):
        loss, ratio, grad = vec(pairs), vec(pairs), vec(rows)
        B.preference_loss(logp, y.to(index), vocab, torch.tensor(o, dtype=offset_type, device="cuda"), 0.1, loss, grad_logp=grad, ref_logp=ref if use_ref else None,
                          pair_weight=w if use_w else None, margin=margin, label_smoothing=smooth, average=average, log_ratio=ratio)
        diff = (logp.double() - (ref.double() if use_ref else 0)).cpu().where(counts, torch.zeros((), dtype=torch.float64)).requires_grad_()
        want, ratios = [], []
        for p in range(pairs):
            s = [diff[o[i]:o[i + 1]].sum() / (max(1, int(counts[o[i]:o[i + 1]].sum())) if average else 1) for i in (2 * p, 2 * p + 1)]
            ratios.append(s[0] - s[1])
            h = 0.1 * ratios[-1] - margin
            each = -(1 - smooth) * torch.nn.functional.logsigmoid(h) - smooth * torch.nn.functional.logsigmoid(-h)
            want.append(each * (float(w[p]) if use_w else 1.0))
        sum(want).backward()
        # sums in 64 bits, one rounding to float each
        close(ratio.cpu(), torch.stack(ratios).detach(), 2.0 ** -23 * torch.stack(ratios).detach().abs() + 1e-12, "log_ratio")
        close(loss.cpu(), torch.stack(want).detach(), 2.0 ** -23 * torch.stack(want).detach().abs() + 1e-12, "loss")
        slope = diff.grad.where(counts, torch.zeros((), dtype=torch.float64))
        close(grad.cpu(), slope, 2.0 ** -23 * slope.abs() + 1e-12, "grad_logp")
        only = vec(pairs)
        B.preference_loss(logp, y.to(index), vocab, torch.tensor(o, dtype=offset_type, device="cuda"), 0.1, only, ref_logp=ref if use_ref else None,
                          pair_weight=w if use_w else None, margin=margin, label_smoothing=smooth, average=average)
        assert torch.equal(only, loss)


def test_preference_takes_what_logp_lacks():
    """Log-probabilities of -10 to the last digit of 64 bits: in float alone the mean of 1000 of them would be 2^-21 off at worst."""
    rows = 1000
    exact = -10 - torch.rand(rows, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    logp = exact.float()
    rest = (exact - logp.double()).float()
    y, o = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.tensor([0, 999, 1000], device="cuda")
    loss, ratio = vec(1), vec(1)
    B.preference_loss(logp, y, 9, o, 1.0, loss, average=True, log_ratio=ratio, logp_rest=rest)
    want = exact[:999].mean() - exact[999]
    close(ratio[0], want, 2.0 ** -24 * want.abs() + 2.0 ** -47, "log_ratio")


def test_preference_of_nothing_and_of_offsets_out_of_range():
    grad = vec(4)
    none = torch.empty(0, device="cuda")
    y, logp = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    B.preference_loss(logp, y, 9, torch.zeros(1, dtype=torch.int32, device="cuda"), 0.1, none, grad_logp=grad)
    assert (grad == 0).all()                              # no pairs: no sequence has any row
    B.preference_loss(none, torch.empty(0, dtype=torch.int32, device="cuda"), 9, torch.zeros(3, dtype=torch.int32, device="cuda"), 0.1, loss := vec(1))
    close(loss, torch.tensor([math.log(2)], device="cuda"), 1e-7, "a pair of nothing")
    guard = torch.full((12,), 7.0, device="cuda")
    for o in ([-5, 2, 900], [3, 1, 2], [1 << 40, 0, -(1 << 40)]):
        B.preference_loss(logp, y, 9, torch.tensor(o, dtype=torch.int64, device="cuda"), 0.1, loss, grad_logp=guard[4:8])
        assert (guard[:4] == 7).all() and (guard[8:] == 7).all() and loss.isfinite().all()


def test_preference_of_infinite_margins():
    o = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    y = torch.zeros(2, dtype=torch.int64, device="cuda")
    loss, grad = vec(1), vec(2)
    for logp, want, slope in (([0.0, -INF], 0.0, 0.0), ([-INF, 0.0], INF, -0.5), ([3000.0, 0.0], 0.0, 0.0), ([0.0, 3000.0], 1500.0, -0.5)):
        B.preference_loss(torch.tensor(logp, device="cuda"), y, 9, o, 0.5, loss, grad_logp=grad)
        assert loss.item() == want and grad[0].item() == slope and grad[1].item() == -slope


def test_a_pair_from_logits_to_gradient():
    """The three calls of a preference step against autograd in 64 bits."""
    rows, vocab, o = 40, 701, [3, 20, 37]
    r = Rows(rows, vocab, 0, 0, F32, 1.0)
    ref = (r.logp + normal(4, rows, dtype=F32)).float()
    logp, stats, loss, grad, d = vec(rows), vec(2 * rows).view(rows, 2), vec(1), vec(rows), r.box()
    B.token_logp(r.z.t, r.y, 1.0, logp, stats=stats)
    B.preference_loss(logp, r.y, vocab, torch.tensor(o, device="cuda"), 0.3, loss, grad_logp=grad, ref_logp=ref)
    B.token_logp_backward(r.z.t, r.y, 1.0, stats, grad, d.t)
    z = r.z.t.double().requires_grad_()
    each = torch.where(r.counts, z.log_softmax(1).gather(1, r.safe[:, None])[:, 0] - ref.double(), 0.0)
    want = -torch.nn.functional.logsigmoid(0.3 * (each[o[0]:o[1]].sum() - each[o[1]:o[2]].sum()))
    want.backward()
    close(loss[0], want.detach(), 1e-5, "loss")
    close(d.t, z.grad, 2e-5 * z.grad.abs() + 1e-7, "dlogits")


def test_streams_graphs_and_repetition():
    r = Rows(333, 32000, 0, 0, BF16, 1.0)
    old, ref, adv, weight = policy_inputs(r)
    offsets = torch.tensor([0, 100, 200, 250, 333], device="cuda")

    def buffers():
        return dict(loss=vec(333), d=r.box().t, logp=vec(333), stats=vec(666).view(333, 2), pair=vec(2), grad=vec(333), d2=r.box().t)

    def all_of(b, s):
        B.policy_loss_and_grad(r.z.t, r.y, 1.0, adv, weight, b["loss"], b["d"], old_logp=old, ref_logp=ref, kl_weight=0.1, stream=s)
        B.token_logp(r.z.t, r.y, 1.0, b["logp"], stats=b["stats"], stream=s)
        B.preference_loss(b["logp"], r.y, 32000, offsets, 0.1, b["pair"], grad_logp=b["grad"], ref_logp=ref, stream=s)
        B.token_logp_backward(r.z.t, r.y, 1.0, b["stats"], b["grad"], b["d2"], stream=s)
    first = buffers()
    all_of(first, None)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [buffers() for _ in range(3)]
    for _ in range(4):
        for s, b in zip(streams, got):
            all_of(b, s)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        all_of(got[2], s)
    torch.cuda.synchronize()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for b in got:
        for k in first:
            assert torch.equal(b[k], first[k]), k


def test_offsets_beyond_32_bits():
    rows, vocab, ld = 3, 4097, (1 << 31) + 9
    raw = torch.empty(2 * ld + vocab, dtype=BF16, device="cuda")
    z = raw.as_strided((rows, vocab), (ld, 1))
    z.copy_(normal(1, rows, vocab))
    y, one = torch.tensor([3, 4096, 0], device="cuda"), torch.ones(rows, device="cuda")
    near, far, loss, d = vec(rows), vec(rows), vec(rows), torch.empty(rows, vocab, dtype=BF16, device="cuda")
    stats = vec(2 * rows).view(rows, 2)
    B.token_logp(z.clone(), y, 1.0, near, stats=stats)
    B.token_logp(z, y, 1.0, far)
    assert torch.equal(near, far)
    B.policy_loss_and_grad(z.clone(), y, 1.0, one, one, loss, d)
    B.policy_loss_and_grad(z, y, 1.0, one, one, far, z)
    assert torch.equal(far, loss) and torch.equal(z, d)
