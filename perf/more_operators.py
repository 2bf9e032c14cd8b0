"""Cases of the operators of alignment training: AdamW over many tensors with states in 8 or 32 bits, policy and preference
losses on token log-probabilities, norms after and before a block fused with its gate and scales.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes the inputs on the GPU, ``run``
makes one pass.  With ``own`` false a pass is made of elementary torch operations; with ``own`` true it makes the calls a
user makes of this package.  ``exact`` computes the same results from the operators' definitions in 64 bits.
"""
import math
import random

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0            # largest finite value of the 8-bit format (4 exponent bits, 3 mantissa bits)
E4M3_LEAST = 2.0 ** -9      # its smallest positive value
BLOCK = 256                 # elements that share a scale
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.1
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INDEX = {"int32": torch.int32, "int64": torch.int64}
ACTIVATIONS = ("none", "sigmoid", "silu")


def listed():
    return [
        # adapters or a small head: a handful of small tensors, one of them of a single element
        dict(name="adam 8 bits, 9 small tensors", op="adam", tensors=9, largest=65537, sizes=1, state="e4m3", rest="none", clip=False),
        # a student's worth of ragged tensors, parameters as bfloat16 pairs, gradients clipped to a norm
        dict(name="adam 8 bits, 120 ragged, clipped", op="adam", tensors=120, largest=8388613, sizes=2, state="e4m3", rest="bf16", clip=True),
        # four layers of LLaMA-7B, bfloat16 pairs: what one GPU of eight holds of a sharded state
        dict(name="adam 8 bits, 4 LLaMA-7B layers", op="adam", layers=4, state="e4m3", rest="bf16", clip=False),
        # one layer with float states and master weights, clipped
        dict(name="adam 32 bits, 1 LLaMA-7B layer", op="adam", layers=1, state="f32", rest="f32", clip=True),
        # a handful of sampled tokens with GPT-2's vocabulary (odd: rows are not aligned), logits in 32 bits
        dict(name="policy 5 x 50257 f32", op="policy", rows=5, vocab=50257, dtype="f32", index="int64", temperature=1.0, old=True, ref=True),
        # a batch of sampled tokens with LLaMA-7B's vocabulary
        dict(name="policy 4096 x 32000", op="policy", rows=4096, vocab=32000, dtype="bf16", index="int32", temperature=0.7, old=True, ref=True),
        # one pair of short answers
        dict(name="preference 1 pair, 61 x 32000 f32", op="preference", rows=61, vocab=32000, pairs=1, dtype="f32", index="int64", temperature=1.0, average=True),
        # a batch of pairs with GPT-2's vocabulary: log-probabilities, the pairs' loss, the gradient of the logits
        dict(name="preference 8 pairs, 2049 x 50257", op="preference", rows=2049, vocab=50257, pairs=8, dtype="bf16", index="int64", temperature=1.0, average=False),
        # scoring one generated token under a large vocabulary
        dict(name="logp 1 x 131071", op="logp", rows=1, vocab=131071, dtype="bf16", index="int64", temperature=1.0),
        # one new token of a 4096-wide model between two blocks, output in 8 bits for the next product
        dict(name="block norm 1 token to 8 bits", op="blocknorm", rows=1, cols=4096, gate="channel", act="none", out="e4m3", backward=False),
        # a training batch of the same width, odd number of tokens, a learned gate for each channel, forward and backward
        dict(name="block norm train 8191 x 4096", op="blocknorm", rows=8191, cols=4096, gate="channel", act="none", out="bf16", backward=True),
        # a batch of a wider model whose gate is computed for each token
        dict(name="block norm train 2047 x 5120 gated", op="blocknorm", rows=2047, cols=5120, gate="token", act="sigmoid", out="bf16", backward=True),
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of `step`, uniform in the logarithm over [lo, hi]."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + step)))
    return max(lo, min(hi, int(v) // step * step))


def draw(rng):
    op = rng.choice(["adam", "adam", "policy", "preference", "logp", "blocknorm", "blocknorm"])
    if op == "adam":
        state = rng.choice(["e4m3", "e4m3", "f32"])
        return dict(op=op, tensors=_log_int(rng, 1, 160), largest=_log_int(rng, 1000, 1 << 23), sizes=rng.randrange(1 << 20), state=state,
                    rest=rng.choice(["none", "bf16", "bf16", "f32"]), clip=rng.random() < 0.5)
    if op == "blocknorm":
        backward, whole = rng.random() < 0.6, rng.random() < 0.8            # widths of models are multiples of 8; some are not
        return dict(op=op, rows=_log_int(rng, 1, 8191), cols=_log_int(rng, 64, 8192, 8) if whole else _log_int(rng, 65, 4095),
                    gate=rng.choice(["none", "channel", "token"]), act=rng.choice(ACTIVATIONS), out="bf16" if backward else rng.choice(["bf16", "e4m3"]),
                    backward=backward)
    vocab = _log_int(rng, 1000, 131072)
    rows = _log_int(rng, 2, min(8192, 130_000_000 // vocab))
    case = dict(op=op, rows=rows, vocab=vocab, dtype=rng.choice(["bf16", "bf16", "f32"]), index=rng.choice(["int32", "int64"]), temperature=rng.choice([0.7, 1.0, 1.3]))
    if op == "policy":
        case.update(old=rng.random() < 0.8, ref=rng.random() < 0.7)
    elif op == "preference":
        case.update(pairs=_log_int(rng, 1, max(1, min(64, rows // 2))), average=rng.random() < 0.3)
    return case


# ------------------------------------------------------------------------------------------------------------ inputs ---

def _sizes(case):
    if "layers" in case:          # LLaMA-7B: four attention projections, three of the feed-forward block, two norms a layer
        return ([4096 * 4096] * 4 + [4096 * 11008] * 3 + [4096] * 2) * case["layers"]
    r = random.Random(case["sizes"])
    return [case["largest"]] + [_log_int(r, 1, case["largest"]) for _ in range(case["tensors"] - 1)]


def _normal(g, shape, std, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _stream_values(g, rows, cols):
    """A residual stream: unit scale, a few channels far larger than the rest."""
    x = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.float32)
    big = torch.rand(cols, generator=g, device="cuda") < 1 / 128
    return (x * torch.where(big, 24.0, 1.0)).to(torch.bfloat16)


def _prepare_adam(s, case, g):
    """All tensors of a kind are views of one buffer, each beginning on a multiple of BLOCK; what lies between them is zero."""
    sizes = _sizes(case)
    begins, total = [], 0
    for n in sizes:
        begins.append(total)
        total += -(-n // BLOCK) * BLOCK
    there = torch.ones(total, dtype=torch.bool, device="cuda")
    for at, n in zip(begins, sizes):
        there[at + n:at + -(-n // BLOCK) * BLOCK] = False

    def new(std, dtype):
        return _normal(g, (total,), std, torch.float32).mul_(there).to(dtype)

    master = new(0.02, torch.float32)
    s["theta"] = master.to(torch.bfloat16)
    s["rest"] = {"none": None, "bf16": (master - s["theta"].float()).to(torch.bfloat16), "f32": master}[case["rest"]]
    s["grad"] = new(1e-3, torch.bfloat16)
    m, r = new(3e-4, torch.float32), new(1e-3, torch.float32).abs_()
    if case["state"] == "f32":
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, r * r, None, None
    else:
        for name, t in (("m", m), ("v", r)):
            t = t.view(-1, BLOCK)
            scale = t.abs().amax(1) / E4M3_MAX
            s[name] = torch.where(scale[:, None] > 0, t / scale[:, None], 0.0).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scale"] = scale
    s["step"], s["seed"], s["max_norm"] = 99, 0x123456789ABCDEF, 1.0
    s["norm"], s["grad_scale"] = torch.zeros(1, device="cuda"), torch.ones(1, device="cuda")
    s["spans"] = list(zip(begins, sizes))


def _prepare_logits(s, case, g):
    rows, vocab, tau = case["rows"], case["vocab"], case["temperature"]
    z = torch.randn((rows, vocab), generator=g, device="cuda").mul_(2.0)
    s["logits"] = z.to(DTYPES[case["dtype"]])
    z = s["logits"].float().div_(tau)
    noise = torch.rand(z.shape, generator=g, device="cuda").clamp_min_(1e-30).log_().neg_().clamp_min_(1e-30).log_().neg_()
    target = (z + noise).argmax(1)                  # sampled from the model
    del noise
    logp = z.gather(1, target[:, None])[:, 0] - torch.logsumexp(z, 1)
    pick = torch.rand(rows, generator=g, device="cuda")
    masked = (pick < 0.1) & (torch.arange(rows, device="cuda") > 0)      # prompts and padding
    s["target"] = torch.where(masked, -1, target).to(INDEX[case["index"]])
    noisy = lambda std: torch.where(masked, 0.0, logp + std * torch.randn(rows, generator=g, device="cuda"))  # noqa: E731
    s["old_logp"], s["ref_logp"] = noisy(0.15), noisy(0.4)
    f32 = lambda *n: torch.empty(n, dtype=torch.float32, device="cuda")  # noqa: E731
    s["logp"], s["dlogits"], s["grad_logp"] = f32(rows), torch.empty_like(s["logits"]), f32(rows)
    if case["op"] == "policy":
        s["advantage"] = torch.randn(rows, generator=g, device="cuda")
        weight = (torch.rand(rows, generator=g, device="cuda") < 0.9).float()
        weight[0] = 1.0
        s["row_weight"] = weight / weight.sum()
        s["loss"], s["kl"] = f32(rows), f32(rows) if case["ref"] else None
    elif case["op"] == "preference":
        cuts = 2 * case["pairs"] - 1
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.randint(0, rows + 1, (cuts,), generator=g, device="cuda").sort().values,
                                  torch.full((1,), rows, dtype=torch.int64, device="cuda")]).to(torch.int32)
        s["pair_weight"] = torch.full((case["pairs"],), 1.0 / case["pairs"], device="cuda")
        s["stats"], s["loss"], s["log_ratio"] = f32(rows, 2), f32(case["pairs"]), f32(case["pairs"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "adam":
        _prepare_adam(s, case, g)
    elif case["op"] != "blocknorm":
        _prepare_logits(s, case, g)
    else:
        rows, cols = case["rows"], case["cols"]
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        weight = lambda: (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(torch.bfloat16)  # noqa: E731
        s["x"], s["block"] = _stream_values(g, rows, cols), _normal(g, (rows, cols), 0.5)
        s["post"], s["pre"] = weight(), weight()
        s["gate"] = None if case["gate"] == "none" else _normal(g, (1 if case["gate"] == "channel" else rows, cols), 1.0)
        s["residual_scale"], s["block_scale"] = 0.9, 0.3
        s["r"], s["rstd_post"], s["rstd_pre"] = new(rows, cols), new(rows, dtype=torch.float32), new(rows, dtype=torch.float32)
        if case["out"] == "e4m3":
            s["y8"], s["scale"] = new(rows, cols, dtype=torch.float8_e4m3fn), new(rows, dtype=torch.float32)
        else:
            s["y"] = new(rows, cols)
        if case["backward"]:
            s["dy"], s["dr"] = _normal(g, (rows, cols), 1e-3), _normal(g, (rows, cols), 1e-3)
            s["dx"], s["dblock"], s["dpost"], s["dpre"] = new(rows, cols), new(rows, cols), new(cols), new(cols)
            s["dgate"] = None if s["gate"] is None else torch.empty_like(s["gate"])
    return s


# -------------------------------------------------------------------------------------------------------- plain forms ---

M32 = 0xFFFFFFFF


def _mix(x):
    """32 bits to 32 bits; of a Python int or of an int64 tensor."""
    x = ((x ^ (x >> 16)) * 0x6A09E667) & M32
    x = ((x ^ (x >> 15)) * 0xB504F333) & M32
    return x ^ (x >> 16)


def _key(seed, step):
    k = _mix(step >> 32)
    for word in (step & M32, seed >> 32, seed & M32):
        k = _mix((word + k) & M32)
    return k


def _dither(key, begin, count):
    """16 random bits for each of the plan's positions [begin, begin + count) as a fraction in [0, 1)."""
    p = torch.arange(begin // 2, (begin + count) // 2, dtype=torch.int64, device="cuda")
    h = _mix(((p & M32) + _mix(((p >> 32) + key) & M32)) & M32)
    return torch.stack((h & 0xFFFF, h >> 16), 1).view(-1).float() * 2.0 ** -16


def _plain_scale(t):
    """Codes before rounding, and the scale, of blocks [n, BLOCK]."""
    most = t.abs().amax(1, keepdim=True)
    most = torch.where(most < 2.0 ** -100, 0.0, most)
    return torch.where(most > 0, t * (E4M3_MAX / torch.where(most > 0, most, 1.0)), 0.0), most / E4M3_MAX


def _plain_root_codes(r, dither):
    u, scale = _plain_scale(r)
    u = torch.where(u > 0, u.clamp_min(E4M3_LEAST), u)
    step = torch.exp2((torch.frexp(u).exponent - 1).clamp_min(-6).float() - 3)
    q = (torch.floor(u / step + dither) * step).clamp_max(E4M3_MAX)
    return q.to(torch.float8_e4m3fn), scale


def _nearest_bf16(x):
    """The bfloat16 values nearest to 64-bit ones.  (By way of a float that is rounded to odd: rounded twice to nearest, ties would go astray.)"""
    f = x.float()
    bits = f.view(torch.int32)
    wide = f.double()
    bits = torch.where(wide.abs() > x.abs(), bits - 1, bits) | (wide != x)
    return bits.view(torch.float32).to(torch.bfloat16)


def _plain_adam(s):
    case = s["case"]
    s["step"] += 1
    t, out = s["step"], {}
    g = s["grad"].float()
    if case["clip"]:
        norm = torch.sqrt((g * g).sum(dtype=torch.float64))
        s["norm"].copy_(norm)
        s["grad_scale"].copy_((s["max_norm"] / norm).clamp_max(1.0))
        g = g * s["grad_scale"]
        out["norm"] = s["norm"]
    if case["state"] == "f32":
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square_()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    del g
    root = torch.sqrt(v)
    delta = (m * (1 / (1 - BETA1 ** t))) / (root * (1 / math.sqrt(1 - BETA2 ** t)) + ADAM_EPS)
    if case["rest"] == "f32":
        x = s["rest"]
        x.add_(-LR * (delta + DECAY * x))
        s["theta"].copy_(x)
    elif case["rest"] == "bf16":            # (a pair holds more bits than a float: in 64)
        x = s["theta"].double().add_(s["rest"])
        x.add_(delta.double().add_(x, alpha=DECAY), alpha=-LR)
        s["theta"].copy_(_nearest_bf16(x))
        s["rest"].copy_(x.sub_(s["theta"]))
    else:
        x = s["theta"].float()
        s["theta"].copy_(x - LR * (delta + DECAY * x))
    del x, delta
    if case["state"] == "f32":
        s["m"], s["v"] = s["m"].copy_(m), s["v"].copy_(v)
    else:
        u, scale = _plain_scale(m.view(-1, BLOCK))
        s["m"].copy_(u.to(torch.float8_e4m3fn).view(-1))
        s["m_scale"].copy_(scale[:, 0])
        q, scale = _plain_root_codes(root.view(-1, BLOCK), _dither(_key(s["seed"], t), 0, root.numel()).view(-1, BLOCK))
        s["v"].copy_(q.view(-1))
        s["v_scale"].copy_(scale[:, 0])
    return _adam_outputs(s, out)


def _adam_outputs(s, out):
    out.update({n: s[n] for n in ("theta", "rest", "m", "v", "m_scale", "v_scale") if s[n] is not None})
    return out


def _plain_logp(s):
    """Exponentials of the logits relative to the row's largest, their sum, log-probabilities (64 bits), and which rows count."""
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    e = torch.exp((z - top) / s["case"]["temperature"])
    total = e.sum(1, keepdim=True)
    target = s["target"].long()
    counts = (target >= 0) & (target < s["case"]["vocab"])
    at = torch.where(counts, target, 0)[:, None]
    logp = (z.gather(1, at) - top).double()[:, 0] / s["case"]["temperature"] - torch.log(total.double())[:, 0]
    return e, total, torch.where(counts, logp, 0.0), counts, at


def _plain_dlogits(s, e, total, at, coef):
    """Gradient of the logits from that of the log-probabilities."""
    coef = (coef / s["case"]["temperature"]).float()[:, None]
    d = -coef * (e / total)
    d.scatter_add_(1, at, coef)
    return torch.where(coef != 0, d, 0.0).to(s["logits"].dtype)


CLIP_LOW, CLIP_HIGH, KL_WEIGHT = 0.2, 0.28, 0.04
BETA, MARGIN, SMOOTHING = 0.1, 0.05, 0.1


def _plain_policy(s):
    case = s["case"]
    e, total, logp, counts, at = _plain_logp(s)
    a, w = s["advantage"], torch.where(counts, s["row_weight"], 0.0)
    ratio = torch.exp(logp - s["old_logp"]) if case["old"] else torch.ones_like(logp)
    free, held = ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    loss, coef = -torch.minimum(free, held), torch.where(free <= held, -free, 0.0)
    out = {}
    if case["ref"]:
        d = torch.where(counts, s["ref_logp"] - logp, 0.0)
        out["kl"] = torch.expm1(d) - d
        loss, coef = loss + KL_WEIGHT * out["kl"], coef - KL_WEIGHT * torch.expm1(d)
        out["kl"] = torch.where(w != 0, out["kl"], 0.0).float()
    out["loss"], out["logp"] = torch.where(w != 0, w * loss, 0.0).float(), torch.where(w != 0, logp, 0.0).float()
    out["dlogits"] = _plain_dlogits(s, e, total, at, torch.where(w != 0, w * coef, 0.0))
    return out


def _plain_preference(s):
    case = s["case"]
    e, total, logp, counts, at = _plain_logp(s)
    offsets, w = s["offsets"].long(), s["pair_weight"].double()
    each = torch.where(counts, logp - s["ref_logp"], 0.0)
    sums = torch.cat([each.new_zeros(1), each.cumsum(0)])
    number = torch.cat([counts.new_zeros(1, dtype=torch.int64), counts.cumsum(0)])
    sums, number = sums[offsets[1:]] - sums[offsets[:-1]], number[offsets[1:]] - number[offsets[:-1]]
    per = 1.0 / number.clamp_min(1) if case["average"] else torch.ones_like(sums)
    sums = (sums * per).view(-1, 2)
    log_ratio = sums[:, 0] - sums[:, 1]
    h = BETA * log_ratio - MARGIN
    soft = lambda x: torch.log1p(torch.exp(-x.abs())) + torch.clamp(x, min=0)  # noqa: E731
    loss = w * ((1 - SMOOTHING) * soft(-h) + SMOOTHING * soft(h))
    dh = w * (SMOOTHING / (1 + torch.exp(-h)) - (1 - SMOOTHING) / (1 + torch.exp(h)))
    of_sequence = (BETA * torch.stack((dh, -dh), 1).view(-1)) * per
    row_sequence = torch.searchsorted(offsets[1:].contiguous(), torch.arange(case["rows"], device="cuda"), right=True)
    grad = torch.where(counts, of_sequence[row_sequence], 0.0)
    return {"logp": logp.float(), "log_ratio": log_ratio.float(), "loss": loss.float(), "grad_logp": grad.float(),
            "dlogits": _plain_dlogits(s, e, total, at, grad)}


def _act_and_slope(name, g):
    if name == "none":
        return g, torch.ones_like(g)
    sig = 1 / (1 + torch.exp(-g))
    return (sig, sig * (1 - sig)) if name == "sigmoid" else (g * sig, sig * (1 + g * (1 - sig)))


def _plain_blocknorm(s):
    case, x, o = s["case"], s["x"].float(), s["block"].float()
    post, pre = s["post"].float(), s["pre"].float()
    rstd_post = torch.rsqrt((o * o).mean(1, keepdim=True) + EPS)
    n = o * rstd_post
    act, slope = (1.0, None) if s["gate"] is None else _act_and_slope(case["act"], s["gate"].float())
    r = s["residual_scale"] * x + s["block_scale"] * act * (n * post)
    rstd_pre = torch.rsqrt((r * r).mean(1, keepdim=True) + EPS)
    y = r * rstd_pre * pre
    out = {"r": r.to(torch.bfloat16)}
    if case["out"] == "e4m3":
        out["scale"] = y.abs().amax(1) / E4M3_MAX
        out["y8"] = torch.where(out["scale"][:, None] > 0, y / out["scale"][:, None], 0.0).to(torch.float8_e4m3fn)
    else:
        out["y"] = y.to(torch.bfloat16)
    if case["backward"]:
        dy, nr = s["dy"].float(), r * rstd_pre
        g = dy * pre
        dr = rstd_pre * (g - nr * (g * nr).mean(1, keepdim=True)) + s["dr"].float()
        out["dpre"] = (dy * nr).sum(0)
        out["dx"] = s["residual_scale"] * dr
        u = s["block_scale"] * dr
        if s["gate"] is not None:
            out["dgate"] = u * (n * post)
            if case["gate"] == "channel":
                out["dgate"] = out["dgate"].sum(0, keepdim=True)
            out["dgate"] = out["dgate"] * slope
        dn = u * act
        out["dpost"] = (dn * n).sum(0)
        h = dn * post
        out["dblock"] = rstd_post * (h - n * (h * n).mean(1, keepdim=True))
        out.update({k: v.to(torch.bfloat16) for k, v in out.items() if k[0] == "d"})
    return out


# --------------------------------------------------------------------------------------------------------------- runs ---

def _own(s):
    from paper_2405_03637_b200 import binding as B
    case = s["case"]
    op = case["op"]
    if op == "adam":
        if "plan" not in s:                     # a training program makes it once
            def views(name, per=1):
                t = s[name]
                return [None if t is None else t[at // per:at // per + -(-n // per)] for at, n in s["spans"]]
            s["plan"] = B.adam_plan_create(list(zip(views("theta"), views("rest"), views("m"), views("v"), views("m_scale", BLOCK),
                                                    views("v_scale", BLOCK), views("grad"))))
            s["workspace"] = torch.empty(B.workspace_bytes(), dtype=torch.uint8, device="cuda")
            B.workspace_init(s["workspace"])
        s["step"] += 1
        if case["clip"]:
            B.adam_grad_norm(s["plan"], s["max_norm"], s["norm"], s["grad_scale"], s["workspace"])
        B.adam_step(s["plan"], B.make_hyper(LR, BETA1, BETA2, ADAM_EPS, DECAY), s["step"], seed=s["seed"], grad_scale=s["grad_scale"] if case["clip"] else None)
        return _adam_outputs(s, {"norm": s["norm"]} if case["clip"] else {})
    if op == "policy":
        B.policy_loss_and_grad(s["logits"], s["target"], case["temperature"], s["advantage"], s["row_weight"], s["loss"], s["dlogits"],
                               old_logp=s["old_logp"] if case["old"] else None, ref_logp=s["ref_logp"] if case["ref"] else None,
                               clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_weight=KL_WEIGHT if case["ref"] else 0.0, logp=s["logp"], kl=s["kl"])
        return {n: s[n] for n in ("kl", "loss", "logp", "dlogits") if s[n] is not None}
    if op == "logp":
        B.token_logp(s["logits"], s["target"], case["temperature"], s["logp"])
        return {"logp": s["logp"]}
    if op == "preference":
        if "logp_rest" not in s:                # what rounding the log-probabilities to float takes, which a sequence's sum adds up
            s["logp_rest"] = torch.empty_like(s["logp"])
        B.token_logp(s["logits"], s["target"], case["temperature"], s["logp"], stats=s["stats"], logp_rest=s["logp_rest"])
        B.preference_loss(s["logp"], s["target"], case["vocab"], s["offsets"], BETA, s["loss"], s["grad_logp"], ref_logp=s["ref_logp"],
                          pair_weight=s["pair_weight"], margin=MARGIN, label_smoothing=SMOOTHING, average=case["average"], log_ratio=s["log_ratio"],
                          logp_rest=s["logp_rest"])
        B.token_logp_backward(s["logits"], s["target"], case["temperature"], s["stats"], s["grad_logp"], s["dlogits"])
        return {n: s[n] for n in ("logp", "log_ratio", "loss", "grad_logp", "dlogits")}
    act = (B.GATE_NONE, B.GATE_SIGMOID, B.GATE_SILU)[ACTIVATIONS.index(case["act"])]
    scales = dict(eps=EPS, residual_scale=s["residual_scale"], block_scale=s["block_scale"], activation=act)
    B.block_norm(s["x"], s["block"], s["r"], gate=s["gate"], post_weight=s["post"], pre_weight=s["pre"], y=s.get("y"), y8=s.get("y8"),
                 y8_scale=s.get("scale"), rstd_post=s["rstd_post"], rstd_pre=s["rstd_pre"], **scales)
    out = {n: s[n] for n in ("r", "y", "y8", "scale") if s.get(n) is not None}
    if case["backward"]:
        if "workspace" not in s:                # scratch that a training program allocates once
            s["workspace"] = torch.empty(B.block_norm_workspace_bytes(case["cols"]), dtype=torch.uint8, device="cuda")
        B.block_norm_backward(s["dy"], None, s["block"], s["rstd_post"], s["rstd_pre"], s["dx"], s["dblock"], dr=s["dr"], gate=s["gate"],
                              post_weight=s["post"], pre_weight=s["pre"], dgate=s["dgate"], dpost_weight=s["dpost"], dpre_weight=s["dpre"],
                              workspace=s["workspace"], residual_scale=s["residual_scale"], block_scale=s["block_scale"], activation=act,
                              x=s["x"])     # (still there: r has an array of its own)
        out.update({n: s[n] for n in ("dx", "dblock", "dpost", "dpre", "dgate") if s[n] is not None})
    return out


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "adam":
        return _plain_adam(state)
    if op == "policy":
        return _plain_policy(state)
    if op == "logp":
        return {"logp": _plain_logp(state)[2].float()}
    return _plain_preference(state) if op == "preference" else _plain_blocknorm(state)


def work(case):
    if case["op"] == "adam":
        n = sum(_sizes(case))
        rest = {"none": 0, "bf16": 4, "f32": 8}[case["rest"]]
        theta = 2 if case["rest"] == "f32" else 4               # with a master weight it is written only
        state = 16 if case["state"] == "f32" else 4 + 16 / BLOCK
        return {"bytes": n * (2 + theta + rest + state), "flops": (18 + (2 if case["clip"] else 0)) * n}
    if case["op"] == "blocknorm":
        n, c = case["rows"] * case["cols"], case["cols"]
        gate = {"none": 0, "channel": 2 * c, "token": 2 * n}[case["gate"]]
        b = 4 * n + 4 * c + gate + 2 * n + (n + 4 * case["rows"] if case["out"] == "e4m3" else 2 * n)
        if case["backward"]:
            b += 4 * n + 4 * n + 4 * c + gate
        return {"bytes": b, "flops": (30 if case["backward"] else 10) * n}
    n, size = case["rows"] * case["vocab"], 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"] * (4 + (4 if case["index"] == "int32" else 8))
    if case["op"] == "logp":
        return {"bytes": n * size + rows, "flops": 4 * n}
    return {"bytes": 2 * n * size + rows + 24 * case["rows"], "flops": 8 * n}


# -------------------------------------------------------------------------------------------- the definitions, 64 bits ---

def _exact_codes(u):
    """Nearest e4m3 values (ties to even) of |u| <= 448 in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(u / step) * step


def _exact_dither(key, begin, count):
    """The definition's random fractions, from 16-bit halves."""
    mask = 0xFFFFFFFF

    def times(x, c):                             # modulo 2^32 without leaving 63 bits
        lo, hi = x & 0xFFFF, x >> 16
        return (lo * c + (((hi * c) & 0xFFFF) << 16)) & mask

    def mixed(x):
        x = times(x.bitwise_xor(x >> 16), 0x6A09E667)
        x = times(x.bitwise_xor(x >> 15), 0xB504F333)
        return x.bitwise_xor(x >> 16)

    at = torch.arange(begin, begin + count, dtype=torch.int64, device="cuda")
    pair = torch.div(at, 2, rounding_mode="floor")
    h = mixed((pair.remainder(2 ** 32) + mixed((torch.div(pair, 2 ** 32, rounding_mode="floor") + key) & mask)) & mask)
    return torch.where(at % 2 == 1, torch.div(h, 65536, rounding_mode="floor"), h.remainder(65536)).double() / 65536


def _exact_adam(s):
    case, t, total = s["case"], s["step"] + 1, s["theta"].numel()
    d = lambda n, a, b: s[n][a:b].double()  # noqa: E731
    part = 1 << 26
    out, gscale = {}, 1.0
    if case["clip"]:
        sq = sum(float(d("grad", a, a + part).square().sum()) for a in range(0, total, part))
        out["norm"] = torch.tensor([math.sqrt(sq)], dtype=torch.float64)
        gscale = min(1.0, s["max_norm"] / math.sqrt(sq))
    got = {n: [] for n in ("theta", "rest", "m", "v", "m_scale", "v_scale") if s[n] is not None}
    key = _key(s["seed"], t)
    for a in range(0, total, part):
        b = min(total, a + part)
        g, m, v = d("grad", a, b) * gscale, d("m", a, b), d("v", a, b)
        if case["state"] == "e4m3":
            m = m * d("m_scale", a // BLOCK, b // BLOCK).repeat_interleave(BLOCK)
            v = (v * d("v_scale", a // BLOCK, b // BLOCK).repeat_interleave(BLOCK)) ** 2
        m, v = m * BETA1 + g * (1 - BETA1), v * BETA2 + g ** 2 * (1 - BETA2)
        x = d("rest", a, b) if case["rest"] == "f32" else d("theta", a, b) + (d("rest", a, b) if case["rest"] == "bf16" else 0)
        x = x * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
        if case["rest"] == "bf16":              # a pair: the nearest value and what it lacks
            scale = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -126))) - 7)      # a bfloat16's spacing there
            near = torch.round(x / scale) * scale
            del scale
            got["theta"].append(near)
            got["rest"].append(x - near)
        else:
            got["theta"].append(x)
            if case["rest"] == "f32":
                got["rest"].append(x)
        if case["state"] == "f32":
            got["m"].append(m)
            got["v"].append(v)
            continue
        for name, w in (("m", m), ("v", v.sqrt())):
            w = w.view(-1, BLOCK)
            scale = w.abs().max(dim=1).values / E4M3_MAX
            u = torch.nan_to_num(w / scale.unsqueeze(1))
            if name == "m":
                got["m"].append(_exact_codes(u).view(-1))
            else:
                u = torch.where(u > 0, u.clamp_min(E4M3_LEAST), u)
                spacing = torch.exp2(torch.floor(torch.log2(u.clamp_min(2.0 ** -6))) - 3)
                near = torch.round(u / spacing)
                scaled = torch.where((u / spacing - near).abs() < 1e-12, near, u / spacing)      # the block's largest is 448 itself
                got["v"].append((torch.floor(scaled + _exact_dither(key, a, b - a).view(-1, BLOCK)) * spacing).clamp_max(E4M3_MAX).view(-1))
            got[name + "_scale"].append(scale)
    out.update({n: torch.cat(v) for n, v in got.items()})
    return out


def _exact_tokens(s, case):
    tau, rows = case["temperature"], case["rows"]
    z = s["logits"].to(torch.float64).div_(tau)
    lse = torch.logsumexp(z, 1)
    target = s["target"].to(torch.int64)
    counts = target.ge(0)
    safe = target.clamp(min=0)
    logp = (z[torch.arange(rows, device="cuda"), safe] - lse).masked_fill(~counts, 0.0)
    if case["op"] == "logp":
        return {"logp": logp}
    if case["op"] == "policy":
        a, w = s["advantage"].double(), s["row_weight"].double() * counts
        ratio = (logp - s["old_logp"].double()).exp() if case["old"] else torch.ones_like(logp)
        over = ((a > 0) & (ratio > 1 + CLIP_HIGH)) | ((a < 0) & (ratio < 1 - CLIP_LOW))
        loss = -a * torch.where(over, torch.where(a > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW), ratio)
        coef = torch.where(over, 0.0, -a * ratio)
        out = {"logp": logp * (w != 0)}
        if case["ref"]:
            k = (s["ref_logp"].double() - logp).masked_fill(~counts, 0.0)
            kl = torch.special.expm1(k) - k
            loss, coef = loss + KL_WEIGHT * kl, coef + KL_WEIGHT * (1 - k.exp())
            out["kl"] = kl * (w != 0)
        out["loss"], coef = w * loss, w * coef
    else:
        edge = s["offsets"].tolist()
        w, coef, out = s["pair_weight"].tolist(), torch.zeros_like(logp), {"logp": logp}
        diff = (logp - s["ref_logp"].double()).masked_fill(~counts, 0.0)
        losses, ratios = [], []
        for p in range(case["pairs"]):
            spans = [slice(edge[2 * p], edge[2 * p + 1]), slice(edge[2 * p + 1], edge[2 * p + 2])]
            div = [max(1, int(counts[i].sum())) if case["average"] else 1 for i in spans]
            ratios.append(float(diff[spans[0]].sum()) / div[0] - float(diff[spans[1]].sum()) / div[1])
            h = torch.tensor(BETA * ratios[-1] - MARGIN, dtype=torch.float64)
            losses.append(w[p] * float(-(1 - SMOOTHING) * torch.nn.functional.logsigmoid(h) - SMOOTHING * torch.nn.functional.logsigmoid(-h)))
            slope = w[p] * BETA * float(torch.sigmoid(h) - (1 - SMOOTHING))
            coef[spans[0]], coef[spans[1]] = slope / div[0], -slope / div[1]
        coef = coef * counts
        out.update(log_ratio=torch.tensor(ratios, dtype=torch.float64), loss=torch.tensor(losses, dtype=torch.float64), grad_logp=coef)
    grad = z.sub_(lse.unsqueeze(1)).exp_().neg_()
    grad[torch.arange(rows, device="cuda"), safe] += 1
    out["dlogits"] = grad.mul_((coef / tau).unsqueeze(1))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adam":
        return _exact_adam(s)
    if case["op"] != "blocknorm":
        return _exact_tokens(s, case)
    d = lambda n: s[n].to(torch.float64)  # noqa: E731
    x, o, post, pre = d("x"), d("block"), d("post"), d("pre")
    norm = lambda t: torch.sqrt(t.pow(2).sum(1, keepdim=True) / case["cols"] + EPS)  # noqa: E731
    rms_o = norm(o)
    n = o / rms_o
    if s["gate"] is None:
        act = slope = torch.ones((), dtype=torch.float64, device="cuda")
    else:
        gate = d("gate")
        sig = torch.sigmoid(gate)
        act, slope = {"none": (gate, torch.ones_like(gate)), "sigmoid": (sig, sig * torch.sigmoid(-gate)),
                      "silu": (gate * sig, sig + gate * sig * torch.sigmoid(-gate))}[case["act"]]
    alpha, beta = s["residual_scale"], s["block_scale"]
    r = alpha * x + beta * act * n * post
    rms_r = norm(r)
    nr = r / rms_r
    y = nr * pre
    out = {"r": r}
    if case["out"] == "e4m3":
        out["scale"] = y.abs().max(dim=1).values / E4M3_MAX
        out["y8"] = _exact_codes(torch.nan_to_num(y / out["scale"].unsqueeze(1)))
    else:
        out["y"] = y
    if case["backward"]:
        dot = lambda a, b: torch.einsum("rc,rc->r", a, b).unsqueeze(1) / case["cols"]  # noqa: E731
        dy = d("dy")
        out["dpre"] = torch.einsum("rc,rc->c", dy, nr)
        dr = (dy * pre - nr * dot(dy * pre, nr)) / rms_r + d("dr")
        out["dx"] = alpha * dr
        dn = beta * dr * act
        out["dpost"] = torch.einsum("rc,rc->c", dn, n)
        out["dblock"] = (dn * post - n * dot(dn * post, n)) / rms_o
        if s["gate"] is not None:
            dgate = beta * dr * n * post * slope
            out["dgate"] = dgate.sum(0, keepdim=True) if case["gate"] == "channel" else dgate
    return out
