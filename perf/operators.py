"""Cases of the training-side operators: residual RMS norm, 8-bit row quantisation, gated feed-forward, distillation loss.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes the inputs on the GPU, ``run``
makes one pass.  With ``own`` false a pass is made of elementary torch operations in 32 bits; with ``own`` true it makes the
calls a user makes of this package.  ``exact`` computes the same results from the operators' definitions in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5
E4M3_MAX = 448.0            # largest finite value of the 8-bit format (4 exponent bits, 3 mantissa bits)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INDEX = {"int32": torch.int32, "int64": torch.int64}


def listed():
    return [
        # one new token of a 4096-wide model (LLaMA-7B's width): residual added, output in 8 bits for the next product
        dict(name="norm 1 token to 8 bits", op="norm", rows=1, cols=4096, residual=True, out="e4m3", backward=False),
        # a training batch of the same width, odd number of tokens, forward and backward
        dict(name="norm train 8191 x 4096", op="norm", rows=8191, cols=4096, residual=True, out="bf16", backward=True),
        # the activations of a small decode batch, rounded before the down projection
        dict(name="quantise 37 x 11008", op="quantize", rows=37, cols=11008),
        # one projection's weights after an optimizer step, for an evaluation in 8 bits
        dict(name="quantise 11008 x 4096", op="quantize", rows=11008, cols=4096),
        # one new token through LLaMA-7B's feed-forward projections: the weights are read once
        dict(name="gated 1 token", op="gated", rows=1, cols=4096, ffn=11008, act="silu", backward=False),
        # a short ragged batch of a GPT-2-small-wide model, forward and backward, with the other activation
        dict(name="gated train 333 x 768", op="gated", rows=333, cols=768, ffn=2048, act="gelu_tanh", backward=True),
        # a training batch through LLaMA-7B's feed-forward projections, forward and backward
        dict(name="gated train 8192 x 4096", op="gated", rows=8192, cols=4096, ffn=11008, act="silu", backward=True),
        # a decode batch through the same projections in 8 bits
        dict(name="gated 8 bits 16 tokens", op="gated8", rows=16, cols=4096, ffn=11008, act="silu"),
        # a prompt (or an evaluation batch), odd number of tokens
        dict(name="gated 8 bits 4095 tokens", op="gated8", rows=4095, cols=4096, ffn=11008, act="silu"),
        # a handful of positions with GPT-2's vocabulary (odd: rows are not aligned) in 32 bits, loss and gradient in one call
        dict(name="distill 7 x 50257 f32", op="distill", rows=7, vocab=50257, k=8, temperature=1.0, dtype="f32", index="int64", fused=True),
        # a training batch with LLaMA-7B's vocabulary, loss and gradient in one call
        dict(name="distill 4096 x 32000", op="distill", rows=4096, vocab=32000, k=64, temperature=2.0, dtype="bf16", index="int32", fused=True),
        # the same with GPT-2's vocabulary and the backward pass in a call of its own, as an autograd engine makes it
        dict(name="distill 2049 x 50257 split", op="distill", rows=2049, vocab=50257, k=21, temperature=1.5, dtype="bf16", index="int64", fused=False),
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of `step`, uniform in the logarithm over [lo, hi]."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + step)))
    return max(lo, min(hi, int(v) // step * step))


def draw(rng):
    op = rng.choice(["norm", "quantize", "gated", "gated", "gated8", "distill", "distill"])
    if op == "norm":
        backward = rng.random() < 0.6
        return dict(op=op, rows=_log_int(rng, 1, 8192), cols=_log_int(rng, 64, 8192, 8) if rng.random() < 0.8 else _log_int(rng, 65, 8191),
                    residual=rng.random() < 0.7, out="bf16" if backward else rng.choice(["bf16", "e4m3"]), backward=backward)
    if op == "quantize":
        return dict(op=op, rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 64, 11008, 8) if rng.random() < 0.8 else _log_int(rng, 65, 11007))
    if op == "gated":          # widths of models are multiples of 8, numbers of tokens are not
        return dict(op=op, rows=_log_int(rng, 1, 8192), cols=_log_int(rng, 128, 4096, 8), ffn=_log_int(rng, 256, 11008, 8),
                    act=rng.choice(["silu", "gelu_tanh"]), backward=rng.random() < 0.6)
    if op == "gated8":
        return dict(op=op, rows=_log_int(rng, 1, 8192), cols=_log_int(rng, 128, 4096, 16), ffn=_log_int(rng, 256, 11008, 16),
                    act=rng.choice(["silu", "gelu_tanh"]))
    vocab = _log_int(rng, 1000, 131072)
    rows = _log_int(rng, 1, min(8192, 160_000_000 // vocab))
    return dict(op=op, rows=rows, vocab=vocab, k=_log_int(rng, 1, 256), temperature=rng.choice([0.7, 1.0, 2.0, 4.0]),
                dtype=rng.choice(["bf16", "bf16", "f32"]), index=rng.choice(["int32", "int64"]), fused=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------------------ inputs ---

def _normal(g, shape, std, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _stream_values(g, rows, cols):
    """A residual stream: unit scale, a few channels far larger than the rest."""
    x = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.float32)
    big = torch.rand(cols, generator=g, device="cuda") < 1 / 128
    return (x * torch.where(big, 24.0, 1.0)).to(torch.bfloat16)


def _in_8_bits(t):
    """Values and one scale a row: what a program that keeps 8-bit weights and activations has in hand."""
    f = t.float()
    scale = f.abs().amax(1) / E4M3_MAX
    return (f / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, s = case["op"], dict(case=case)
    new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if op == "norm":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _stream_values(g, rows, cols)
        s["residual"] = _stream_values(g, rows, cols) if case["residual"] else None
        s["weight"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(torch.bfloat16)
        s["r"] = new(rows, cols) if case["residual"] else None
        if case["out"] == "e4m3":
            s["y8"], s["scale"] = new(rows, cols, dtype=torch.float8_e4m3fn), new(rows, dtype=torch.float32)
        else:
            s["y"] = new(rows, cols)
        if case["backward"]:
            s["dy"] = _normal(g, (rows, cols), 1e-3)
            s["dr"] = _normal(g, (rows, cols), 1e-3) if case["residual"] else None
            s["rstd"], s["dx"], s["dweight"] = new(rows, dtype=torch.float32), new(rows, cols), new(cols)
    elif op == "quantize":
        s["x"] = _normal(g, (case["rows"], case["cols"]), 0.02)
        s["q"], s["scale"] = new(case["rows"], case["cols"], dtype=torch.float8_e4m3fn), new(case["rows"], dtype=torch.float32)
    elif op in ("gated", "gated8"):
        rows, cols, ffn = case["rows"], case["cols"], case["ffn"]
        s["x"], s["w_gate"], s["w_up"] = _normal(g, (rows, cols), 1.0), _normal(g, (ffn, cols), 0.02), _normal(g, (ffn, cols), 0.02)
        s["h"] = new(rows, ffn)
        if op == "gated8":
            for name in ("x", "w_gate", "w_up"):
                s[name], s[name + "_scale"] = _in_8_bits(s[name])
        elif case["backward"]:
            s["dh"] = _normal(g, (rows, ffn), 1e-3)
            s["gate"], s["up"], s["dgate"], s["dup"] = new(rows, ffn), new(rows, ffn), new(rows, ffn), new(rows, ffn)
            s["dx"], s["dw_gate"], s["dw_up"] = new(rows, cols), new(ffn, cols), new(ffn, cols)
    else:
        rows, vocab, k = case["rows"], case["vocab"], case["k"]
        z = torch.randn((rows, vocab), generator=g, device="cuda").mul_(2.0)
        s["logits"] = z.to(DTYPES[case["dtype"]])
        top, index = torch.topk(z.add_(torch.randn(z.shape, generator=g, device="cuda")), k, dim=1)
        # some rows have fewer entries than k, some have none, some weigh nothing (prompts and padding)
        kept = torch.randint(1, k + 1, (rows, 1), generator=g, device="cuda")
        pick = torch.rand((rows, 1), generator=g, device="cuda")
        kept = torch.where(pick < 0.8, k, torch.where(pick < 0.95, kept, 0))
        index = torch.where(torch.arange(k, device="cuda") < kept, index, -1)
        s["index"], s["top"] = index.to(INDEX[case["index"]]), top.contiguous()
        weight = (torch.rand(rows, generator=g, device="cuda") < 0.9).float()
        weight[0] = 1.0
        s["row_weight"] = weight / weight.sum()
        s["loss"], s["dlogits"] = new(rows, dtype=torch.float32), torch.empty_like(s["logits"])
        if not case["fused"]:
            s["lse"] = new(rows, dtype=torch.float32)
    return s


# --------------------------------------------------------------------------------------------------------- plain form ---

def _act_and_slope(name, g):
    """Activation and its derivative."""
    if name == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_quantize(y):
    scale = y.abs().amax(1) / E4M3_MAX
    q = torch.where(scale[:, None] > 0, y / scale[:, None], torch.zeros_like(y))
    return q.to(torch.float8_e4m3fn), scale


def _plain_norm(s):
    r = s["x"].float()
    out = {}
    if s["residual"] is not None:
        r = r + s["residual"].float()
        out["r"] = r.to(torch.bfloat16)
    rstd = torch.rsqrt((r * r).mean(1, keepdim=True) + EPS)
    w = s["weight"].float()
    y = r * rstd * w
    if s["case"]["out"] == "e4m3":
        out["y8"], out["scale"] = _plain_quantize(y)
    else:
        out["y"] = y.to(torch.bfloat16)
    if s["case"]["backward"]:
        dy = s["dy"].float()
        n = r * rstd
        wdy = w * dy
        dx = rstd * (wdy - n * (wdy * n).mean(1, keepdim=True))
        if s["dr"] is not None:
            dx = dx + s["dr"].float()
        out["dx"], out["dweight"] = dx.to(torch.bfloat16), (dy * n).sum(0).to(torch.bfloat16)
    return out


def _plain_gated(s):
    case = s["case"]
    x, wg, wu = (s[n].float() for n in ("x", "w_gate", "w_up"))
    if case["op"] == "gated8":
        x, wg, wu = (t * s[n + "_scale"][:, None] for t, n in ((x, "x"), (wg, "w_gate"), (wu, "w_up")))
    gate, up = x @ wg.T, x @ wu.T
    a, slope = _act_and_slope(case["act"], gate)
    out = {"h": (a * up).to(torch.bfloat16)}
    if case.get("backward"):
        dh = s["dh"].float()
        dgate, dup = dh * up * slope, dh * a
        out["dx"] = (dgate @ wg + dup @ wu).to(torch.bfloat16)
        out["dw_gate"], out["dw_up"] = (dgate.T @ x).to(torch.bfloat16), (dup.T @ x).to(torch.bfloat16)
    return out


def _plain_distill(s):
    case = s["case"]
    tau = case["temperature"]
    z = s["logits"].float() / tau
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    index = s["index"].long()
    there = index >= 0
    t = torch.where(there, s["top"] / tau, -math.inf)
    most = t.amax(1, keepdim=True)
    any_there = most > -math.inf
    shifted = t - torch.where(any_there, most, 0.0)
    pe = torch.where(there, torch.exp(shifted), 0.0)
    psum = torch.where(any_there, pe.sum(1, keepdim=True), 1.0)
    p = pe / psum
    at = index.clamp_min(0)
    logq = z.gather(1, at) - lse
    terms = torch.where(p > 0, p * (shifted - torch.log(psum) - logq), 0.0)
    loss = torch.where(any_there[:, 0], tau * tau * terms.sum(1), 0.0)
    dz = tau * torch.where(any_there, e / total, 0.0)
    dz.scatter_add_(1, at, -tau * p)
    weight = s["row_weight"]
    dz = torch.where(weight[:, None] != 0, weight[:, None] * dz, 0.0)
    out = {"dlogits": dz.to(s["logits"].dtype)}
    if case["fused"]:
        out["loss"] = weight * loss
    else:
        out["loss"], out["lse"] = loss, lse[:, 0]
    return out


# --------------------------------------------------------------------------------------------------------------- runs ---

def _own(s):
    from paper_2405_03637_b200 import binding as B
    case = s["case"]
    op = case["op"]
    if op == "norm":
        B.add_rms_norm(s["x"], s["residual"], s["weight"], EPS, residual_out=s["r"], y=s.get("y"), y8=s.get("y8"),
                       y8_scale=s.get("scale"), rstd=s.get("rstd"))
        out = {n: s[n] for n in ("r", "y", "y8", "scale") if s.get(n) is not None}
        if case["backward"]:
            if "workspace" not in s:            # scratch that a training program allocates once
                s["workspace"] = torch.empty(B.rms_norm_workspace_bytes(case["cols"]), dtype=torch.uint8, device="cuda")
            B.add_rms_norm_backward(s["dy"], s["x"] if s["r"] is None else s["r"], s["rstd"], s["weight"], s["dx"], s["dweight"],
                                    s["workspace"], dresidual=s["dr"])
            out["dx"], out["dweight"] = s["dx"], s["dweight"]
        return out
    if op == "quantize":
        B.quantize_rows(s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if op in ("gated", "gated8"):
        act = B.ACT_SILU if case["act"] == "silu" else B.ACT_GELU_TANH
        if op == "gated8":
            B.gated_ffn_e4m3(s["x"], s["x_scale"], s["w_gate"], s["w_gate_scale"], s["w_up"], s["w_up_scale"], s["h"], act)
            return {"h": s["h"]}
        B.gated_ffn(s["x"], s["w_gate"], s["w_up"], s["h"], gate=s.get("gate"), up=s.get("up"), activation=act)
        if not case["backward"]:
            return {"h": s["h"]}
        B.gated_ffn_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], s["gate"], s["up"], s["dgate"], s["dup"], dx=s["dx"],
                             dw_gate=s["dw_gate"], dw_up=s["dw_up"], activation=act)
        return {n: s[n] for n in ("h", "dx", "dw_gate", "dw_up")}
    if case["fused"]:
        B.distill_loss_and_grad(s["logits"], s["index"], s["top"], case["temperature"], s["row_weight"], s["loss"], s["dlogits"])
        return {n: s[n] for n in ("dlogits", "loss")}
    B.distill_loss(s["logits"], s["index"], s["top"], case["temperature"], s["loss"], lse=s["lse"])
    B.distill_loss_backward(s["logits"], s["index"], s["top"], case["temperature"], s["lse"], s["row_weight"], s["dlogits"])
    return {n: s[n] for n in ("dlogits", "loss", "lse")}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "norm":
        return _plain_norm(state)
    if op == "quantize":
        q, scale = _plain_quantize(state["x"].float())
        return {"q": q, "scale": scale}
    return _plain_gated(state) if op in ("gated", "gated8") else _plain_distill(state)


def work(case):
    op, rows = case["op"], case["rows"]
    if op == "norm":
        n, c = rows * case["cols"], case["cols"]
        b = 2 * n + 2 * c + (4 * n if case["residual"] else 0) + (n + 4 * rows if case["out"] == "e4m3" else 2 * n)
        if case["backward"]:
            b += 4 * n + (2 * n if case["residual"] else 0) + 2 * c
        return {"bytes": b, "flops": (16 if case["backward"] else 6) * n}
    if op == "quantize":
        n = rows * case["cols"]
        return {"bytes": 3 * n + 4 * rows, "flops": 3 * n}
    if op in ("gated", "gated8"):
        c, f = case["cols"], case["ffn"]
        if op == "gated8":
            return {"bytes": rows * c + 2 * c * f + 4 * (rows + 2 * f) + 2 * rows * f, "flops": 4 * rows * c * f}
        b = 2 * (rows * c + 2 * c * f + rows * f)
        if case["backward"]:
            return {"bytes": b + 2 * (rows * f + rows * c + 2 * c * f), "flops": 12 * rows * c * f}
        return {"bytes": b, "flops": 4 * rows * c * f}
    n, size = rows * case["vocab"], 2 if case["dtype"] == "bf16" else 4
    entry = 4 + (4 if case["index"] == "int32" else 8)
    return {"bytes": 2 * n * size + rows * (case["k"] * entry + 8), "flops": 8 * n}


# -------------------------------------------------------------------------------------------- the definitions, 64 bits ---

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    d = lambda n: s[n].to(torch.float64)  # noqa: E731

    def to_8_bits(y):
        scale = y.abs().max(dim=1).values / E4M3_MAX
        u = torch.nan_to_num(y / scale.unsqueeze(1))
        # nearest multiple of the spacing at |u|: 2^(e-3) for 2^e <= |u| < 2^(e+1), not below 2^-9 (ties to even)
        e = torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6)))
        step = torch.exp2(e - 3)
        return torch.round(u / step) * step, scale

    if op == "quantize":
        q, scale = to_8_bits(d("x"))
        return {"q": q, "scale": scale}
    if op == "norm":
        r = d("x") + (d("residual") if case["residual"] else 0)
        rms = torch.sqrt(r.pow(2).sum(1, keepdim=True) / case["cols"] + EPS)
        n = r / rms
        y = n * d("weight")
        out = {"r": r} if case["residual"] else {}
        if case["out"] == "e4m3":
            out["y8"], out["scale"] = to_8_bits(y)
        else:
            out["y"] = y
        if case["backward"]:
            dn = d("dy") * d("weight")
            out["dweight"] = torch.einsum("rc,rc->c", d("dy"), n)
            out["dx"] = (dn - n * (torch.einsum("rc,rc->r", dn, n) / case["cols"]).unsqueeze(1)) / rms + (d("dr") if case["residual"] else 0)
        return out
    if op in ("gated", "gated8"):
        x, wg, wu = d("x"), d("w_gate"), d("w_up")
        if op == "gated8":
            x, wg, wu = x * d("x_scale").unsqueeze(1), wg * d("w_gate_scale").unsqueeze(1), wu * d("w_up_scale").unsqueeze(1)
        gate, up = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
        if case["act"] == "silu":
            a = gate * torch.sigmoid(gate)
            slope = torch.sigmoid(gate) + a * torch.sigmoid(-gate)
        else:
            inner = math.sqrt(2 / math.pi) * (gate + 0.044715 * gate.pow(3))
            half = torch.sigmoid(2 * inner)                       # (1 + tanh(inner)) / 2
            a = gate * half
            slope = half + 2 * gate * half * torch.sigmoid(-2 * inner) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * gate.pow(2))
        out = {"h": a * up}
        if case.get("backward"):
            dgate, dup = d("dh") * slope * up, d("dh") * a
            out["dx"] = torch.matmul(dgate, wg) + torch.matmul(dup, wu)
            out["dw_gate"], out["dw_up"] = torch.matmul(dgate.t(), x), torch.matmul(dup.t(), x)
        return out
    tau, rows = case["temperature"], case["rows"]
    z = d("logits").div_(tau)
    lse = torch.logsumexp(z, 1)
    index = s["index"].to(torch.int64)
    absent = index.lt(0)
    t = (d("top") / tau).masked_fill_(absent, -math.inf)
    logp = (t - torch.logsumexp(t, 1, keepdim=True)).nan_to_num_(nan=-math.inf, neginf=-math.inf)
    p = logp.exp()
    safe = index.masked_fill(absent, 0)
    logq = torch.gather(z, 1, safe) - lse.unsqueeze(1)
    loss = tau ** 2 * (p * (logp.masked_fill(absent, 0).nan_to_num(neginf=0.0) - logq)).sum(1)
    mass = p.sum(1)
    grad = (z - lse.unsqueeze(1)).exp_().mul_(mass.unsqueeze(1))
    grad.index_put_((torch.arange(rows, device="cuda").unsqueeze(1).expand_as(safe), safe), -p, accumulate=True)
    grad.mul_((tau * d("row_weight")).unsqueeze(1))
    if case["fused"]:
        return {"dlogits": grad, "loss": loss * d("row_weight")}
    return {"dlogits": grad, "loss": loss, "lse": lse}
