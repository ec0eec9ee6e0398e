"""The framework's learner-side operators at the sizes they are used at: layer norm, the gated feed-forward block and the
orthogonalised update, each in a plain form (elementary torch operations in fp32) and through the framework's own calls."""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5                                       # layer norm
NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)      # quintic iteration
NS_STEPS, NS_EPS = 5, 1e-7

# the largest drawn case costs no more than the largest listed one of its operator
LN_MOST = 16384 * 4096
FFN_MOST = 8192 * 4096 * 16384
NS_MOST = 24 * 1024 * 1024 * 4096


def listed():
    return [
        # one token's row of a small model, where only the latency of a call counts
        {"name": "ln_fwd_token", "op": "ln_fwd", "rows": 1, "width": 512, "pad": 0, "type": "f32"},
        # a large batch of wide activations
        {"name": "ln_fwd_large", "op": "ln_fwd", "rows": 16384, "width": 4096, "pad": 0, "type": "bf16"},
        # a learner's batch of a GPT-2-medium-shaped model, in the type of the gradient vectors
        {"name": "ln_bwd_medium", "op": "ln_bwd", "rows": 4096, "width": 1024, "pad": 0, "type": "f32"},
        # a ragged batch whose width fits no vector load, rows apart by more than the width (a slice of a wider buffer)
        {"name": "ln_bwd_odd", "op": "ln_bwd", "rows": 30011, "width": 2047, "pad": 5, "type": "bf16"},
        # evaluation of a single token: the weights are read once for one row
        {"name": "ffn_fwd_token", "op": "ffn_fwd", "tokens": 1, "width": 1024, "hidden": 4096, "act": "silu", "type": "bf16"},
        # a short ragged prompt through a block of odd sizes
        {"name": "ffn_fwd_ragged", "op": "ffn_fwd", "tokens": 37, "width": 1001, "hidden": 2731, "act": "gelu", "type": "f16"},
        # a large block on a large batch: the tensor cores' rate
        {"name": "ffn_fwd_large", "op": "ffn_fwd", "tokens": 8192, "width": 4096, "hidden": 16384, "act": "silu", "type": "bf16"},
        # a learner's training step through a GPT-2-medium-sized block: outputs, input and weight gradients
        {"name": "ffn_step_medium", "op": "ffn_step", "tokens": 4096, "width": 1024, "hidden": 4096, "act": "silu", "type": "bf16"},
        # the same in fp32 at the Transformer-base sizes, gradients in the type that the compression step takes
        {"name": "ffn_step_base_f32", "op": "ffn_step", "tokens": 2048, "width": 512, "hidden": 2048, "act": "silu", "type": "f32"},
        # one small matrix: a chain of dependent products where latency counts
        {"name": "ns_small", "op": "ns", "batch": 1, "rows": 64, "cols": 256, "type": "bf16"},
        # the feed-forward matrices of 24 layers of a GPT-2-medium-shaped model in one call
        {"name": "ns_layers", "op": "ns", "batch": 24, "rows": 1024, "cols": 4096, "type": "bf16"},
        # tall matrices of odd sizes at fp32 accuracy
        {"name": "ns_tall_f32", "op": "ns", "batch": 6, "rows": 2047, "cols": 511, "type": "f32"},
    ]


def _size(rng, low, high):
    """Log-uniform in [low, high]: a third multiples of 64, a third multiples of 8, the rest as they fall."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    unit = rng.choice((1, 8, 64))
    return max(low, min(high, (v + unit // 2) // unit * unit or v))


def draw(rng):
    op = rng.choice(("ln_fwd", "ln_bwd", "ffn_fwd", "ffn_step", "ns"))
    kind = rng.choice(("f32", "f16", "bf16"))
    if op in ("ln_fwd", "ln_bwd"):
        width = _size(rng, 32, 8192)
        rows = _size(rng, 1, max(1, min(65536, LN_MOST // (2 * width))))
        return {"op": op, "rows": rows, "width": width, "pad": rng.choice((0, 0, 3, 64)), "type": kind}
    if op in ("ffn_fwd", "ffn_step"):
        width, hidden = _size(rng, 64, 4096), _size(rng, 128, 16384)
        most = FFN_MOST // (1 if op == "ffn_fwd" else 3) // (width * hidden)
        tokens = _size(rng, 1, max(1, min(8192, most)))
        return {"op": op, "tokens": tokens, "width": width, "hidden": hidden,
                "act": rng.choice(("silu", "gelu", "relu")), "type": kind}
    rows, cols = _size(rng, 16, 2048), _size(rng, 16, 4096)
    small, large = min(rows, cols), max(rows, cols)
    batch = _size(rng, 1, max(1, min(24, NS_MOST // (small * small * large))))
    return {"op": op, "batch": batch, "rows": rows, "cols": cols, "type": kind}


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _rows(gen, case, scale, shift):
    """Activations [rows, width], as a slice of rows that are `pad` elements longer; a few channels are much larger."""
    rows, width = case["rows"], case["width"]
    x = _randn(gen, rows, width + case["pad"])
    x.mul_(scale).add_(shift)
    x[:, ::97] *= 8.0
    return x.to(TYPES[case["type"]])[:, :width]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, kind = case["op"], TYPES[case["type"]]
    s = {"case": case, "op": op}
    if op in ("ln_fwd", "ln_bwd"):
        s["x"] = _rows(gen, case, 1.5, 0.25)
        s["gamma"] = 1.0 + 0.1 * _randn(gen, case["width"])       # fp32: slices of the flat weight vector
        s["beta"] = 0.1 * _randn(gen, case["width"])
        if op == "ln_bwd":
            s["dy"] = _rows(gen, case, 0.02, 0.0)
            x = s["x"].float()                                    # what the forward pass left behind
            mean = x.mean(1)
            s["mean"] = mean
            s["rstd"] = torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)
    elif op in ("ffn_fwd", "ffn_step"):
        t, d, f = case["tokens"], case["width"], case["hidden"]
        s["x"] = _randn(gen, t, d).to(kind)                       # what a layer norm hands over
        s["w_gate"] = (_randn(gen, f, d) / math.sqrt(d)).to(kind)
        s["w_up"] = (_randn(gen, f, d) / math.sqrt(d)).to(kind)
        s["w_down"] = (_randn(gen, d, f) / math.sqrt(f)).to(kind)
        if op == "ffn_step":
            s["dy"] = (0.02 * _randn(gen, t, d)).to(kind)
    else:
        b, m, n = case["batch"], case["rows"], case["cols"]
        # a momentum of averaged sparse gradients: a fifth of the coordinates set, and directions the learners share
        g = _randn(gen, b, m, n)
        g *= torch.rand(b, m, n, generator=gen, device="cuda") < 0.2
        r = min(4, m, n)
        low = _randn(gen, b, m, r) @ _randn(gen, b, r, n)
        g = g + low * (0.5 * math.sqrt(0.2 / r))
        s["update"] = g.mul_(1e-3)
    return s


# ---- plain forms -----------------------------------------------------------------------------------
def _act(name, g):
    """(act(g), act'(g))"""
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if name == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    on = (g > 0).to(g.dtype)
    return g * on, on


def _plain_ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = torch.rsqrt((c * c).mean(1) + EPS)
    y = c * rstd[:, None] * s["gamma"] + s["beta"]
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_ln_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    r = s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * r
    w = dy * s["gamma"]
    dx = r * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _plain_ffn(s, step):
    kind = s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _act(s["case"]["act"], g)
    h = a * u
    out = {"y": (h @ wd.t()).to(kind)}
    if step:
        dy = s["dy"].float()
        dh = dy @ wd
        dg, du = dh * u * slope, dh * a
        out.update(dx=(dg @ wg + du @ wu).to(kind), dw_gate=(dg.t() @ x).to(kind), dw_up=(du.t() @ x).to(kind),
                   dw_down=(dy.t() @ h).to(kind))
    return out


def _plain_ns(s):
    a, b, c = NS_COEFFICIENTS
    x = s["update"]
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        p = x @ x.transpose(1, 2)
        x = a * x + (b * p + c * (p @ p)) @ x
    if tall:
        x = x.transpose(1, 2)
    return {"out": x.to(TYPES[s["case"]["type"]]).contiguous()}


# ---- the framework's calls -------------------------------------------------------------------------
_handle = None


def _ops():
    """The one operator handle that a training program keeps for its life."""
    global _handle
    if _handle is None:
        import paper_2104_11125_b200 as sc
        _handle = sc.Operators()
    return _handle


def _own(s):
    ops, op = _ops(), s["op"]
    if op == "ln_fwd":
        x = s["x"]
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        mean, rstd = torch.empty((2, x.shape[0]), dtype=torch.float32, device=x.device)
        ops.layer_norm(x, s["gamma"], s["beta"], EPS, y, mean, rstd)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "ln_bwd":
        x = s["x"]
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dgamma, dbeta = torch.empty((2, x.shape[1]), dtype=torch.float32, device=x.device)
        ops.layer_norm_backward(s["dy"], x, s["gamma"], s["mean"], s["rstd"], dx, dgamma, dbeta)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op in ("ffn_fwd", "ffn_step"):
        x, wg, wu, wd, act = s["x"], s["w_gate"], s["w_up"], s["w_down"], s["case"]["act"]
        y = torch.empty_like(x)
        if op == "ffn_fwd":
            ops.gated_ffn(x, wg, wu, wd, y, activation=act)
            return {"y": y}
        saved = torch.empty((2, x.shape[0], wg.shape[0]), dtype=x.dtype, device=x.device)
        ops.gated_ffn(x, wg, wu, wd, y, saved=saved, activation=act)
        dx, dwg, dwu, dwd = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(wd)
        ops.gated_ffn_backward(s["dy"], x, wg, wu, wd, saved, dx, dwg, dwu, dwd, activation=act)
        return {"y": y, "dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    g = s["update"]
    out = torch.empty(g.shape, dtype=TYPES[s["case"]["type"]], device=g.device)
    ops.orthogonalise(g, out, steps=NS_STEPS, coefficients=NS_COEFFICIENTS, eps=NS_EPS)
    return {"out": out}


def run(s):
    if own:
        return _own(s)
    op = s["op"]
    if op == "ln_fwd":
        return _plain_ln_fwd(s)
    if op == "ln_bwd":
        return _plain_ln_bwd(s)
    if op == "ns":
        return _plain_ns(s)
    return _plain_ffn(s, op == "ffn_step")


# ---- the definition in 64 bits ---------------------------------------------------------------------
def _exact_ffn(s, step):
    """Through automatic differentiation of the forward formula, so that the gradients are derived apart from the plain form's."""
    leaf = {k: s[k].double().requires_grad_(step) for k in ("x", "w_gate", "w_up", "w_down")}
    with torch.set_grad_enabled(step):
        g = torch.einsum("td,fd->tf", leaf["x"], leaf["w_gate"])
        u = torch.einsum("td,fd->tf", leaf["x"], leaf["w_up"])
        act = s["case"]["act"]
        if act == "silu":
            a = g * torch.sigmoid(g)
        elif act == "gelu":
            a = 0.5 * g * torch.erfc(-g / math.sqrt(2.0))
        else:
            a = g.clamp(min=0.0)
        y = torch.einsum("tf,df->td", a * u, leaf["w_down"])
    out = {"y": y.detach()}
    if step:
        y.backward(s["dy"].double())
        out.update(dx=leaf["x"].grad, dw_gate=leaf["w_gate"].grad, dw_up=leaf["w_up"].grad, dw_down=leaf["w_down"].grad)
    return out


def _exact_ns(s):
    """The iteration acts on singular values alone: the polynomial on the eigenvalues of the smaller Gram matrix gives one
    factor, applied once. x p(x^2) per step, so the whole is G Q diag(f(s) / s) Q^T."""
    a, b, c = NS_COEFFICIENTS
    g = s["update"].double()
    tall = g.shape[1] > g.shape[2]
    if not tall:
        g = g.transpose(1, 2)
    g = g / (torch.linalg.vector_norm(g, dim=(1, 2), keepdim=True) + NS_EPS)
    lam, q = torch.linalg.eigh(g.transpose(1, 2) @ g)
    lam = lam.clamp(min=0.0)
    factor = torch.ones_like(lam)
    for _ in range(NS_STEPS):
        now = lam * factor.square()
        factor = factor * (a + now * (b + c * now))
    x = g @ ((q * factor[:, None, :]) @ q.transpose(1, 2))
    return {"out": x if tall else x.transpose(1, 2).contiguous()}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "ns":
        return _exact_ns(s)
    if op in ("ffn_fwd", "ffn_step"):
        return _exact_ffn(s, op == "ffn_step")
    x = s["x"].double()
    if op == "ln_fwd":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (x - mean[:, None]) * rstd[:, None] * s["gamma"].double() + s["beta"].double()
        return {"y": y, "mean": mean, "rstd": rstd}
    # the backward pass takes mean and rstd as they are given
    dy, n = s["dy"].double(), case["width"]
    mean, r = s["mean"].double()[:, None], s["rstd"].double()[:, None]
    xh = (x - mean) * r
    p = dy * s["gamma"].double()
    dx = (r / n) * (n * p - p.sum(1, keepdim=True) - xh * torch.einsum("ij,ij->i", p, xh)[:, None])
    return {"dx": dx, "dgamma": torch.einsum("ij,ij->j", dy, xh), "dbeta": torch.einsum("ij->j", dy)}


def work(case):
    op, e = case["op"], {"f32": 4, "f16": 2, "bf16": 2}[case["type"]]
    if op in ("ln_fwd", "ln_bwd"):
        n = case["rows"] * case["width"]
        planes = 2 if op == "ln_fwd" else 3
        return {"bytes": planes * n * e + 8 * case["rows"] + 8 * case["width"] + (8 * case["width"] if op == "ln_bwd" else 0),
                "flops": (8 if op == "ln_fwd" else 14) * n}
    if op in ("ffn_fwd", "ffn_step"):
        t, d, f = case["tokens"], case["width"], case["hidden"]
        if op == "ffn_fwd":
            return {"bytes": e * (2 * t * d + 3 * d * f), "flops": 6 * t * d * f}
        return {"bytes": e * (4 * t * d + 6 * d * f), "flops": 18 * t * d * f}
    b, m, n = case["batch"], case["rows"], case["cols"]
    m, n = min(m, n), max(m, n)
    # both Gram products are symmetric: half of each
    return {"bytes": b * m * n * (4 + e), "flops": NS_STEPS * b * (m * m * n + m * m * m + 2 * m * m * n)}
