"""The multi-tensor AdamW step with states in 8 and 32 bits, and the gradients' norm.

Float states with a parameter alone or a master weight: bit for bit what the flat step with float states computes.  Everything else
against the formulas in 64 bits.  Tolerances: the step's float operations (about ten, two of them approximations of 2 units) put an
update within 2^-20 of itself; a code is half a spacing (2^-4 of the value, 2^-10 of the scale below 2^-6 of it) off, a root's code less
than a whole one, and exactly the one that the documented random bits give unless the sum is within 2^-10 of an integer.
"""
import math

import pytest
import torch

from ops_util import BF16, E4M3, F32, close, normal
from paper_2405_03637_b200 import binding as B

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
M32 = 0xFFFFFFFF
GROUP = 256


def hyper(flags=0, **kw):
    h = {**HYPER, **kw}
    return B.make_hyper(h["lr"], h["beta1"], h["beta2"], h["eps"], h["weight_decay"], flags)


def mix(x):
    x = ((x ^ (x >> 16)) * 0x6A09E667) & M32
    x = ((x ^ (x >> 15)) * 0xB504F333) & M32
    return x ^ (x >> 16)


def dither(seed, step, first, n):
    key = mix(step >> 32)
    for word in (step & M32, seed >> 32, seed & M32):
        key = mix((word + key) & M32)
    p = first + torch.arange(n, dtype=torch.int64, device="cuda")
    h = mix(((p >> 1 & M32) + mix(((p >> 33) + key) & M32)) & M32)
    return torch.where(p % 2 == 1, h >> 16, h & 0xFFFF).double() / 65536


class Guarded:
    """A contiguous vector at an offset inside a buffer of sentinel bytes."""

    def __init__(self, n, dtype, shift=0, data=None):
        size = torch.empty(0, dtype=dtype).element_size()
        self.lo, self.hi = 256 + shift * size, 256 + (shift + n) * size
        self.raw = torch.full((self.hi + 256,), 0x5B, dtype=torch.uint8, device="cuda")
        self.t = self.raw[self.lo:self.hi].view(dtype)
        if data is not None:
            self.t.copy_(data)

    def intact(self):
        return bool((self.raw[:self.lo] == 0x5B).all() and (self.raw[self.hi:] == 0x5B).all())


def codes_of(t):
    """Nearest codes and scales of a vector."""
    n, groups = t.numel(), -(-t.numel() // GROUP)
    pad = torch.zeros(groups * GROUP, device="cuda")
    pad[:n] = t
    scale = pad.view(-1, GROUP).abs().amax(1) / 448
    return torch.where(scale[:, None] > 0, pad.view(-1, GROUP) / scale[:, None], 0.0).to(E4M3).view(-1)[:n], scale


class Tensor:
    def __init__(self, n, state, rest, shift=0, seed=0):
        x, r = normal(seed, n, std=0.02, dtype=F32), normal(seed + 2, n, std=1e-3, dtype=F32).abs()
        m = normal(seed + 1, n, std=3e-4, dtype=F32)
        theta = x.to(BF16)
        self.n, self.state, self.rest_kind = n, state, rest
        self.theta = Guarded(n, BF16, shift, theta)
        self.rest = {B.REST_NONE: None, B.REST_BF16: Guarded(n, BF16, shift, x - theta.float()), B.REST_F32: Guarded(n, F32, shift, x)}[rest]
        self.grad = Guarded(n, BF16, shift, normal(seed + 3, n, std=1e-3))
        if state == B.STATE_F32:
            self.m, self.v, self.m_scale, self.v_scale = Guarded(n, F32, shift, m), Guarded(n, F32, shift, r * r), None, None
        else:
            (cm, sm), (cv, sv) = codes_of(m), codes_of(r)
            self.m, self.v = Guarded(n, E4M3, shift, cm), Guarded(n, E4M3, shift, cv)
            self.m_scale, self.v_scale = Guarded(len(sm), F32, 0, sm), Guarded(len(sv), F32, 0, sv)

    def row(self):
        return tuple(g and g.t for g in (self.theta, self.rest, self.m, self.v, self.m_scale, self.v_scale, self.grad))

    def values(self):
        """x, m and sqrt(v) in 64 bits."""
        x = self.theta.t.double()
        if self.rest is not None:
            x = self.rest.t.double() + (x if self.rest_kind == B.REST_BF16 else 0)
        if self.state == B.STATE_F32:
            return x, self.m.t.double(), self.v.t.double().sqrt()
        s = lambda v: v.t.double().repeat_interleave(GROUP)[:self.n]  # noqa: E731
        return x, self.m.t.double() * s(self.m_scale), self.v.t.double() * s(self.v_scale)

    def intact(self):
        return all(g is None or g.intact() for g in (self.theta, self.rest, self.m, self.v, self.m_scale, self.v_scale, self.grad))


def expected(t, step, scale=1.0, inside=False, **kw):
    """x', m', sqrt(v') in 64 bits, and the magnitudes that went into the update and into m'.

    m' = beta1 m + (1 - beta1) g may cancel: its float roundings are 2^-24 of each product and of the sum, so at most 2^-22 of the sum of
    the products' magnitudes, and the update's error goes by that sum too, not by what is left of it.
    """
    h = {**HYPER, **kw}
    x, m, r = t.values()
    g = t.grad.t.double() * scale
    m_size = h["beta1"] * m.abs() + (1 - h["beta1"]) * g.abs()
    m, v = h["beta1"] * m + (1 - h["beta1"]) * g, h["beta2"] * r * r + (1 - h["beta2"]) * g * g
    vhat = v / (1 - h["beta2"] ** step)
    den = (vhat + h["eps"]).sqrt() if inside else vhat.sqrt() + h["eps"]
    delta = -h["lr"] * (m / (1 - h["beta1"] ** step) / den + h["weight_decay"] * x)
    size = h["lr"] * (m_size / (1 - h["beta1"] ** step) / den + h["weight_decay"] * x.abs())
    return x + delta, m, v.sqrt(), size, m_size


def spacing(v, bits):
    """Distance of neighbouring values of `bits` significant bits around |v|."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(1e-300))) - (bits - 1))


def check(t, want, first, seed, step, what):
    x64, m64, r64, size, m_size = want
    n, off = t.n, 2.0 ** -20 * size
    if t.rest_kind == B.REST_BF16:
        hi, lo = t.theta.t.double(), t.rest.t.double()
        near = off + 2.0 ** -23 * (lo.abs() + size)                  # of theta + RN(rest + update)
        assert ((x64 - hi).abs() <= spacing(x64, 8) / 2 + near).all(), what + " theta is the nearest"
        close(hi + lo, x64, near + 2.0 ** -8 * 1.001 * (x64 - hi).abs() + 1e-38, what + " pair")
    elif t.rest_kind == B.REST_F32:
        close(t.rest.t, x64, off + 2.0 ** -23 * x64.abs(), what + " master")
        assert torch.equal(t.theta.t, t.rest.t.to(BF16))
    else:
        close(t.theta.t, x64, off + 2.0 ** -8 * 1.001 * x64.abs() + 1e-38, what + " theta")
    if t.state == B.STATE_F32:
        close(t.m.t, m64, 2.0 ** -22 * m_size, what + " m")
        close(t.v.t, r64 * r64, 2.0 ** -21 * r64 * r64, what + " v")
        return
    groups = -(-n // GROUP)
    pad = lambda v: torch.cat([v, v.new_zeros(groups * GROUP - n)]).view(groups, GROUP)  # noqa: E731
    sm, sv = pad(m64).abs().amax(1) / 448, pad(r64).amax(1) / 448
    close(t.m_scale.t, sm, 2.0 ** -20 * sm, what + " scale of m")
    close(t.v_scale.t, sv, 2.0 ** -20 * sv, what + " scale of the root")
    each = lambda s: s.repeat_interleave(GROUP)[:n]  # noqa: E731
    _, m_got, r_got = t.values()
    close(m_got, m64, 2.0 ** -4 * 1.001 * m64.abs() + each(sm) * 2.0 ** -10 * 1.001 + 2.0 ** -22 * m_size, what + " m")
    u = torch.where(r64 > 0, (r64 / each(sv).clamp_min(1e-300)).clamp_min(2.0 ** -9), 0.0)
    step_of = torch.exp2(torch.floor(torch.log2(u.clamp_min(2.0 ** -6))) - 3)
    place = u / step_of + dither(seed, step, first, n)
    code = (torch.floor(place) * step_of).clamp_max(448)
    got = t.v.t.double()
    undecided = (place - place.round()).abs() < 2.0 ** -10
    assert (undecided | (got == code)).all(), what + " codes of the root"
    assert (torch.where(undecided, ((got - u).abs() <= step_of * (1 + 2.0 ** -10)) | (got == code), True)).all(), what


FORMS = [(s, r) for s in (B.STATE_E4M3, B.STATE_F32) for r in (B.REST_NONE, B.REST_BF16, B.REST_F32)]
SIZES = [1, 2, 7, 8, 255, 256, 257, 511, 4095, 4096, 4097, 70_001, 0, 8192, 300_000]


@pytest.mark.parametrize("state,rest", FORMS)
@pytest.mark.parametrize("shift", [0, 8, 1])
def test_step_matches_definition(state, rest, shift):
    tensors = [Tensor(n, state, rest, shift, seed=10 * i) for i, n in enumerate(SIZES)]
    plan = B.adam_plan_create([t.row() for t in tensors])
    seed = 0xFEDCBA9876543210
    scale = torch.tensor([0.37], device="cuda")
    for step, kw in ((1, {}), (7, dict(eps=1e-4)), (1000, dict(flags=B.FLAG_EPS_INSIDE_SQRT, eps=1e-9)), ((1 << 33) + 5, dict(weight_decay=0.0))):
        flags = kw.pop("flags", 0)
        use = step == 7
        want = [expected(t, step, float(scale) if use else 1.0, bool(flags), **kw) for t in tensors]
        grads = [t.grad.t.clone() for t in tensors]
        B.adam_step(plan, hyper(flags, **kw), step, seed=seed, grad_scale=scale if use else None)
        first = 0
        for t, w, g in zip(tensors, want, grads):
            if t.n:
                check(t, w, first, seed, step, f"n {t.n} step {step}")
            assert t.intact() and torch.equal(t.grad.t, g)
            first += -(-t.n // GROUP) * GROUP
    B.adam_plan_destroy(plan)


@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("shift", [0, 3])
def test_float_states_are_the_flat_steps_bit_for_bit(master, shift):
    rest = B.REST_F32 if master else B.REST_NONE
    tensors = [Tensor(n, B.STATE_F32, rest, shift, seed=10 * i) for i, n in enumerate(SIZES)]
    flat = [[g and g.t.clone() for g in (t.theta, t.rest, t.m, t.v, t.grad)] for t in tensors]
    plan = B.adam_plan_create([t.row() for t in tensors])
    one = torch.ones(1, device="cuda")
    for step in (1, 2, 50):
        flags = B.FLAG_EPS_INSIDE_SQRT if step == 2 else 0
        B.adam_step(plan, hyper(flags), step, grad_scale=one if step == 2 else None)
        for t, (theta, w, m, v, grad) in zip(tensors, flat):
            if t.n:                                      # (the flat step wants pointers, and an empty tensor has none)
                B.adamw_step_fp32(theta, w, m, v, grad, t.n, hyper(flags), step)
            assert torch.equal(t.theta.t.view(torch.int16), theta.view(torch.int16)) and torch.equal(t.m.t, m) and torch.equal(t.v.t, v)
            assert w is None or torch.equal(t.rest.t, w)
    B.adam_plan_destroy(plan)


def test_results_do_not_depend_on_alignment():
    """Whole aligned groups and groups taken element by element: the same bits."""
    for state, rest in FORMS:
        a, b = Tensor(9000, state, rest, 0), Tensor(9000, state, rest, 1)
        for t in (a, b):
            plan = B.adam_plan_create([t.row()])
            for step in (1, 2, 3):
                B.adam_step(plan, hyper(), step, seed=5)
            B.adam_plan_destroy(plan)
        for x, y in zip(a.row(), b.row()):
            assert x is None or torch.equal(x.view(torch.uint8) if x.dtype is E4M3 else x, y.view(torch.uint8) if y.dtype is E4M3 else y)


def test_seed_and_step_change_the_random_bits_and_nothing_else():
    def run(seed, step):
        t = Tensor(4096, B.STATE_E4M3, B.REST_BF16)
        plan = B.adam_plan_create([t.row()])
        B.adam_step(plan, hyper(beta1=0.0, beta2=0.5), step, seed=seed)
        B.adam_plan_destroy(plan)
        return t
    a, b, c = run(1, 3), run(1, 3), run(2, 3)
    assert torch.equal(a.v.t.view(torch.uint8), b.v.t.view(torch.uint8))
    assert not torch.equal(a.v.t.view(torch.uint8), c.v.t.view(torch.uint8))
    for x, y in ((a.theta, c.theta), (a.rest, c.rest), (a.v_scale, c.v_scale)):
        assert torch.equal(x.t, y.t)
    assert torch.equal(a.m.t.view(torch.uint8), c.m.t.view(torch.uint8))


def test_roots_follow_their_mean_where_rounding_to_nearest_would_not_move():
    """A quarter of the elements keeps its gradients (and the group's largest), the others' vanish: their roots have to decay by
    sqrt(beta2) a step.  Each step's rounding is unbiased; of a root of k codes' steps the decay of 2000 steps of beta2 = 0.999 leaves
    e^-1, with a spread per element below one half (a step of a code is at most an eighth), so the mean over 49152 of them is within 5 x 0.5 / sqrt(49152)."""
    n = 1 << 16
    zeros = lambda k, dtype: torch.zeros(k, dtype=dtype, device="cuda")  # noqa: E731
    theta, grad, m, v = zeros(n, BF16), torch.full((n,), 0.5, dtype=BF16, device="cuda"), zeros(n, E4M3), zeros(n, E4M3)
    v_scale = torch.full((n // GROUP,), 0.5 / 448, device="cuda")
    v.copy_(torch.full((n,), 448.0))
    grad[torch.arange(n, device="cuda") % 4 != 0] = 0
    plan = B.adam_plan_create([(theta, None, m, v, zeros(n // GROUP, F32), v_scale, grad)])
    for step in range(1000, 3000):
        B.adam_step(plan, hyper(lr=0.0), step, seed=11)
    B.adam_plan_destroy(plan)
    r = v.double() * v_scale.double().repeat_interleave(GROUP)
    kept, gone = r[::4], r.view(-1, 4)[:, 1:]
    close(kept, torch.full_like(kept, 0.5), 1e-4, "kept")
    assert abs(float(gone.mean()) / 0.5 / math.exp(-1.0) - 1) < 5 * 0.5 / math.sqrt(gone.numel()) + 0.005


def test_groups_of_zeros_tiny_and_non_finite_values():
    n = 5 * GROUP
    t = Tensor(n, B.STATE_E4M3, B.REST_NONE)
    for g in (t.m, t.v):
        g.t.zero_()
    t.m_scale.t.zero_(), t.v_scale.t.zero_()
    grad = t.grad.t
    grad[:GROUP] = 0                                       # nothing at all
    grad[GROUP:2 * GROUP] = 1e-35                          # m below 2^-100, squares below a float's range
    grad[2 * GROUP + 3], grad[3 * GROUP + 5] = math.inf, math.nan
    before = t.theta.t.clone()
    plan = B.adam_plan_create([t.row()])
    B.adam_step(plan, hyper(weight_decay=0.0, eps=1e-8), 1)
    m, v, sm, sv = t.m.t.float(), t.v.t.float(), t.m_scale.t, t.v_scale.t
    assert (m[:2 * GROUP] == 0).all() and (v[:2 * GROUP] == 0).all() and (sm[:2] == 0).all() and (sv[:2] == 0).all()
    assert torch.equal(t.theta.t[:2 * GROUP], before[:2 * GROUP])
    assert sm[2].isnan() and sv[2].isnan() and sm[3].isnan() and sv[3].isnan() and sm[4].isfinite()
    theta = t.theta.t
    assert theta[2 * GROUP + 3].isnan() and theta[3 * GROUP + 5].isnan() and int(theta.isnan().sum()) == 2
    grad.zero_()
    B.adam_step(plan, hyper(), 2)
    assert t.theta.t[2 * GROUP:4 * GROUP].isnan().all() and t.theta.t[4 * GROUP:].isfinite().all() and t.theta.t[:2 * GROUP].isfinite().all()
    B.adam_plan_destroy(plan)


def test_a_root_that_is_not_zero_has_a_code_that_is_not():
    """Else an element whose m is kept would be divided by eps alone at the next step."""
    n = GROUP
    t = Tensor(n, B.STATE_E4M3, B.REST_NONE)
    for g in (t.m, t.v):
        g.t.zero_()
    t.grad.t.fill_(1e-9)
    t.grad.t[0] = 10.0
    plan = B.adam_plan_create([t.row()])
    for step in range(1, 30):
        B.adam_step(plan, hyper(), step, seed=step)
        assert (t.v.t.float() > 0).all()
    B.adam_plan_destroy(plan)


def test_pairs_of_any_size_keep_what_the_update_adds():
    """Updates far below theta, about as large, and far above it; theta' has to be the nearest bfloat16 throughout."""
    n = 1 << 16
    t = Tensor(n, B.STATE_F32, B.REST_BF16)
    t.theta.t.copy_(normal(1, n, dtype=F32) * torch.exp2(torch.randint(-40, 20, (n,), device="cuda").float()))
    t.rest.t.copy_(t.theta.t.float() * 2.0 ** -9 * normal(2, n, dtype=F32).clamp(-1, 1))
    t.theta.t[:64], t.rest.t[:64] = 0, 0
    plan = B.adam_plan_create([t.row()])
    for step in (10, 11, 12):
        want = expected(t, step, weight_decay=0.0)
        B.adam_step(plan, hyper(weight_decay=0.0), step)
        check(t, want, 0, 0, step, f"step {step}")
    B.adam_plan_destroy(plan)


# ------------------------------------------------------------------------------------------------------- norm, streams ---

def workspace():
    ws = torch.empty(B.workspace_bytes(), dtype=torch.uint8, device="cuda")
    B.workspace_init(ws)
    return ws


@pytest.mark.parametrize("shift", [0, 1])
def test_grad_norm(shift):
    tensors = [Tensor(n, B.STATE_F32, B.REST_NONE, shift, seed=10 * i) for i, n in enumerate(SIZES)]
    plan, ws = B.adam_plan_create([t.row() for t in tensors]), workspace()
    norm, scale = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
    base = [t.grad.t.clone() for t in tensors]
    for factor in (1.0, 1e30, 1e-30, 2.0 ** 120, 0.0):
        for t, g in zip(tensors, base):
            t.grad.t.copy_(g.float() * factor)
        want = math.sqrt(sum(float(t.grad.t.double().square().sum()) for t in tensors))
        for limit in (0.5 * want or 1.0, 2 * want or 1.0, math.inf):
            B.adam_grad_norm(plan, limit, norm, scale, ws)
            close(norm[0], torch.tensor(want, dtype=torch.float64, device="cuda"), 2.0 ** -20 * want, f"norm {factor}")     # eight squares in float
            close(scale[0], torch.tensor(min(1.0, limit / want) if want else 1.0, device="cuda"), 2.0 ** -20, f"scale {factor}")
        B.adam_grad_norm(plan, 1.0, norm, None, ws)
    again = norm.clone()
    for bad, of_norm in ((math.inf, math.inf), (math.nan, math.nan)):
        tensors[4].grad.t[3] = bad
        B.adam_grad_norm(plan, 1.0, norm, scale, ws)
        if math.isinf(bad):
            assert norm.item() == math.inf and scale.item() == 0
        else:
            assert norm.isnan() and scale.isnan()
    tensors[4].grad.t[3] = 0
    B.adam_grad_norm(plan, 1.0, norm, scale, ws)
    assert torch.equal(norm, again)
    B.adam_plan_destroy(plan)


def test_empty_plans():
    ws, norm, scale = workspace(), torch.full((1,), 3.0, device="cuda"), torch.full((1,), 3.0, device="cuda")
    for rows in ([], [Tensor(0, B.STATE_E4M3, B.REST_BF16).row()]):
        plan = B.adam_plan_create(rows)
        B.adam_step(plan, hyper(), 1)
        B.adam_grad_norm(plan, 1.0, norm, scale, ws)
        assert norm.item() == 0 and scale.item() == 1
        B.adam_plan_destroy(plan)


def test_refusals_of_a_plan():
    t = Tensor(1000, B.STATE_E4M3, B.REST_BF16)
    plan, ws = B.adam_plan_create([t.row()]), workspace()
    before = [x.clone() for x in t.row()]
    one = torch.ones(1, device="cuda")

    def refused(status, f, *a, **k):
        with pytest.raises(B.CollageError) as e:
            f(*a, **k)
        assert e.value.status == status
    refused(B.ERR_ARG, B.adam_step, plan, hyper(), 0)
    for bad in (dict(lr=-1.0), dict(beta1=1.0), dict(beta2=math.nan), dict(eps=math.inf), dict(weight_decay=-0.1)):
        refused(B.ERR_ARG, B.adam_step, plan, hyper(**bad), 1)
    refused(B.ERR_ARG, B.adam_step, plan, hyper(B.FLAG_TWOSUM_GROW), 1)
    refused(B.ERR_ARG, B.adam_step, plan, B.make_hyper(1e-3, 0.9, 0.999, 1e-8, 0.0, edq_out=ws, workspace=ws), 1)
    refused(B.ERR_ALIAS, B.adam_step, plan, hyper(), 1, grad_scale=t.m_scale.t[1:2])
    for limit in (0.0, -1.0, math.nan):
        refused(B.ERR_ARG, B.adam_grad_norm, plan, limit, one, None, ws)
    refused(B.ERR_NULL, B.adam_grad_norm, plan, 1.0, None, one, ws)
    refused(B.ERR_WORKSPACE, B.adam_grad_norm, plan, 1.0, one, None, None)
    refused(B.ERR_WORKSPACE, B.adam_grad_norm, plan, 1.0, one, None, ws[:-1])
    refused(B.ERR_ALIAS, B.adam_grad_norm, plan, 1.0, one, one, ws)
    refused(B.ERR_ALIAS, B.adam_grad_norm, plan, 1.0, t.v_scale.t[:1], one, ws)
    torch.cuda.synchronize()
    for x, y in zip(before, t.row()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    B.adam_plan_destroy(plan)


def test_streams_graphs_and_repetition():
    def make():
        t = [Tensor(n, B.STATE_E4M3, B.REST_BF16, seed=i) for i, n in enumerate((70_001, 4096, 300))]
        return t, B.adam_plan_create([x.row() for x in t]), workspace(), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")

    def step(of, k, s):
        _, plan, ws, norm, scale = of
        B.adam_grad_norm(plan, 0.01, norm, scale, ws, stream=s)
        B.adam_step(plan, hyper(), k, seed=9, grad_scale=scale, stream=s)
    sets, streams = [make() for _ in range(4)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in (1, 2, 2, 2):
        step(sets[0], k, None)
        for of, s in zip(sets[1:3], streams):
            step(of, k, s)
    step(sets[3], 1, None)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        step(sets[3], 2, s)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for other in sets[1:]:
        assert torch.equal(other[3], sets[0][3]) and torch.equal(other[4], sets[0][4])
        for a, b in zip(sets[0][0], other[0]):
            for x, y in zip(a.row(), b.row()):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    for of in sets:
        B.adam_plan_destroy(of[1])


def test_many_small_tensors_and_many_chunks():
    sizes = [1 + (i * 37) % 600 for i in range(3000)] + [5_000_001]
    tensors = []
    big = {k: torch.zeros(sum(-(-n // GROUP) * GROUP for n in sizes), dtype=d, device="cuda") for k, d in
           (("theta", BF16), ("m", E4M3), ("v", E4M3), ("grad", BF16))}
    scales = [torch.zeros(big["m"].numel() // GROUP, device="cuda") for _ in range(2)]
    big["grad"].copy_(normal(1, big["grad"].numel(), std=1e-3))
    at = 0
    for n in sizes:
        g = -(-n // GROUP)
        cut = lambda k: big[k][at:at + n]  # noqa: E731
        tensors.append((cut("theta"), None, cut("m"), cut("v"), scales[0][at // GROUP:at // GROUP + g], scales[1][at // GROUP:at // GROUP + g], cut("grad")))
        at += g * GROUP
    plan = B.adam_plan_create(tensors)
    B.adam_step(plan, hyper(weight_decay=0.0), 1, seed=3)
    # the first step of zero states moves every parameter by lr against the gradient's sign
    inside = torch.zeros(at, dtype=torch.bool, device="cuda")
    b = 0
    for n in sizes:
        inside[b:b + n] = True
        b += -(-n // GROUP) * GROUP
    want = torch.where(inside, -1e-3 * big["grad"].double().sign() * (big["grad"].double().abs() / (big["grad"].double().abs() + 1e-8)), 0.0)
    close(big["theta"], want, 2.0 ** -8 * 1.01 * want.abs(), "theta")
    assert (big["v"][~inside].float() == 0).all()
    B.adam_plan_destroy(plan)


def test_positions_beyond_33_bits():
    """The random bits change with the upper word of a pair's number, inside a tensor and behind it (and offsets pass 32 bits)."""
    border, n = 1 << 33, (1 << 33) + 9 * GROUP
    zeros = lambda k, dtype: torch.zeros(k, dtype=dtype, device="cuda")  # noqa: E731
    huge = (zeros(n, BF16), None, zeros(n, E4M3), zeros(n, E4M3), zeros(n // GROUP, F32), zeros(n // GROUP, F32), zeros(n, BF16))
    tail, begin = Tensor(3000, B.STATE_E4M3, B.REST_NONE, seed=4), border - 40 * GROUP
    here = Tensor(n - begin, B.STATE_E4M3, B.REST_NONE, seed=9)                       # what the tensor holds around the border
    parts = [huge[0][begin:], None, huge[2][begin:], huge[3][begin:], huge[4][begin // GROUP:], huge[5][begin // GROUP:], huge[6][begin:]]
    for part, value in zip(parts, here.row()):
        if part is not None:
            part.copy_(value)
    plan = B.adam_plan_create([huge, tail.row()])
    want, want_here = expected(tail, 3), expected(here, 3)
    B.adam_step(plan, hyper(), 3, seed=77)
    for part, value in zip(parts, here.row()):
        if part is not None:
            value.copy_(part)
    check(here, want_here, begin, 77, 3, "around")
    check(tail, want, n, 77, 3, "behind")
    assert int((huge[0][:begin] != 0).sum()) == 0
    B.adam_plan_destroy(plan)
    del huge, parts
    torch.cuda.empty_cache()


@pytest.mark.parametrize("state,rest", FORMS)
def test_many_steps_over_many_tiles(state, rest):
    """Blocks that turn over their stages many times, of ragged tensors between: the same as each tensor by itself, step after step."""
    sizes = [3_000_001, 4864 * 148 * 2, 17, 5000, 3840 * 148 * 3 + 256]
    together, apart = ([Tensor(n, state, rest, seed=i) for i, n in enumerate(sizes)] for _ in range(2))
    plan = B.adam_plan_create([t.row() for t in together])
    alone = [B.adam_plan_create([t.row()]) for t in apart]
    for step in range(1, 21):
        B.adam_step(plan, hyper(), step, seed=step)
        for p in alone:
            B.adam_step(p, hyper(), step, seed=step)
    for a, b in zip(together, apart):
        for k, (x, y) in enumerate(zip(a.row(), b.row())):
            # (a root's random bits go by its position in the plan: only the first tensor has the same ones)
            if x is not None and (a is together[0] or state == B.STATE_F32):
                assert torch.equal(x.view(torch.uint8) if x.dtype is E4M3 else x, y.view(torch.uint8) if y.dtype is E4M3 else y), (a.n, k)
        assert a.intact() and all(x is None or x.float().isfinite().all() for x in a.row())
    assert B.pipeline_fault() == 0
    for p in [plan, *alone]:
        B.adam_plan_destroy(p)
