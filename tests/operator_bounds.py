"""The learner-side operators in 64 bits, with elementwise bounds on how far a kernel may be from them.

The bounds come from the rounding model of the operators' documentation alone, by carrying absolute values through the
formulas:

  u       unit roundoff of the element type (fp32 2^-24, fp16 2^-11, bf16 2^-8), for each stated rounding; below an fp16's normal
          range a rounding moves a value by at most 2^-25.
  gamma   relative error of one product sum, against sum |a| |b|.  16-bit operands are exact factors; the tensor core may
          cut a unit in the last place for each 16 terms: (K/16 + 4) 2^-22.  fp32 operands as two fp16 planes carry 22 bits
          each and leave out lo * lo: 3 * 2^-22; the accumulator is cut at most twelve times in a block of 64, and the blocks'
          sums are rounded: 12 * 2^-23 + (K/64 + 1) 2^-23.  Parts of k add at most 32 roundings in either case.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
# largest second derivative of each activation, and largest slope
CURVE = {"silu": 0.5, "gelu": 0.8, "gelu_tanh": 0.85, "relu": 0.0}
SLOPE = {"silu": 1.1, "gelu": 1.13, "gelu_tanh": 1.13, "relu": 1.0}
# relative error of the activation's own evaluation in fp32 (a few units in the last place of each function in it)
ACT_EVAL = 32 * 2.0 ** -24


def product_error(a, b, kind):
    """Bound on the error of a @ b.T for exact operands a [m, k], b [n, k] (64-bit tensors)."""
    k = a.shape[1]
    gamma = (k / 16 + 36) * 2.0 ** -22 if kind != torch.float32 else 3 * 2.0 ** -22 + 12 * 2.0 ** -23 + (k / 64 + 33) * 2.0 ** -23
    e = gamma * (a.abs() @ b.abs().t())
    if kind == torch.float32:            # what the low plane cannot hold of values far below the tensor's largest
        fa, fb = a.abs().max() * 2.0 ** -38, b.abs().max() * 2.0 ** -38
        e = e + fa * b.abs().sum(1)[None, :] + fb * a.abs().sum(1)[:, None]
    return e


def rounding(v, err, kind):
    """Bound after one more rounding to `kind` of a value that is within err of v."""
    return err + U[kind] * (v.abs() + err) + TINY[kind]


def act(name, g):
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        c = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        s = math.sqrt(2 / math.pi)
        t = torch.tanh(s * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * s * (1 + 3 * 0.044715 * g * g)
    return g.clamp(min=0), (g > 0).to(g.dtype)


def ffn(x, wg, wu, wd, name, kind, dy=None, wgrad=None, saved=None):
    """{output: (value, bound)} of the block, and of its gradients when dy is given.  All tensors 64-bit."""
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = product_error(x, wg, kind), product_error(x, wu, kind)
    a, s = act(name, g)
    ea = SLOPE[name] * eg + ACT_EVAL * (a.abs() + g.abs())
    h = a * u
    eh = ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -24 * h.abs()
    eh = rounding(h, eh, kind)
    y = h @ wd.t()
    out = {"y": (y, rounding(y, product_error(h, wd, kind) + eh @ wd.abs().t(), kind))}
    out["saved"] = (torch.stack([g, u]), torch.stack([rounding(g, eg, kind), rounding(u, eu, kind)]))
    if dy is None:
        return out
    # the backward pass works on the g and u that were stored
    eg, eu = rounding(g, eg, kind), rounding(u, eu, kind)
    es = CURVE[name] * eg + ACT_EVAL * (s.abs() + 1)
    if name == "relu":
        es = es + (g.abs() <= eg).to(g.dtype)
    ea = SLOPE[name] * eg + ACT_EVAL * (a.abs() + g.abs())
    eh = rounding(h, ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -24 * h.abs(), kind)
    dh = dy @ wd
    edh = product_error(dy, wd.t(), kind)
    du, dg = dh * a, dh * u * s
    edu = rounding(du, edh * (a.abs() + ea) + dh.abs() * ea + 2.0 ** -23 * du.abs(), kind)
    edg = rounding(dg, edh * (u.abs() + eu) * (s.abs() + es) + dh.abs() * (eu * (s.abs() + es) + u.abs() * es) + 2.0 ** -22 * dg.abs(), kind)
    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + product_error(dg, wg.t(), kind) + product_error(du, wu.t(), kind)
    out["dx"] = (dx, rounding(dx, edx, kind))
    for key, left, eleft in (("dw_gate", dg, edg), ("dw_up", du, edu)):
        v = left.t() @ x
        out[key] = (v, rounding(v, product_error(left.t(), x.t(), kind) + eleft.t() @ x.abs(), wgrad))
    v = dy.t() @ h
    out["dw_down"] = (v, rounding(v, product_error(dy.t(), h.t(), kind) + dy.abs().t() @ eh, wgrad))
    return out


def layer_norm(x, gamma, beta, eps, kind):
    """{output: (value, bound)}; sums of `width` fp32 terms, a few hundred at most one after another, then a tree."""
    n = x.shape[1]
    depth = min(n, 300) + 20
    mean = x.mean(1, keepdim=True)
    em = depth * 2.0 ** -24 * x.abs().mean(1, keepdim=True) + 2.0 ** -24 * mean.abs()
    c = x - mean
    ec = em + 2.0 ** -24 * c.abs()
    var = c.square().mean(1, keepdim=True)
    ev = (2 * c.abs() * ec + ec.square()).mean(1, keepdim=True) + depth * 2.0 ** -24 * var
    rstd = (var + eps).rsqrt()
    er = rstd * (0.5 * ev / (var + eps) * 1.5 + 4 * 2.0 ** -24)
    g = torch.ones(n, dtype=x.dtype, device=x.device) if gamma is None else gamma
    b = torch.zeros(n, dtype=x.dtype, device=x.device) if beta is None else beta
    y = c * rstd * g + b
    ey = (ec * (rstd + er) + c.abs() * er) * g.abs() + 4 * 2.0 ** -24 * ((c * rstd * g).abs() + b.abs())
    return {"y": (y, rounding(y, ey, kind)), "mean": (mean[:, 0], em[:, 0] + 2.0 ** -24 * mean[:, 0].abs()),
            "rstd": (rstd[:, 0], er[:, 0])}


def layer_norm_backward(dy, x, gamma, mean, rstd, kind):
    """mean and rstd as given (64-bit copies of what the operator is given)."""
    rows, n = x.shape
    depth, deep = min(n, 300) + 20, min(rows, 2000) + 300
    e = 2.0 ** -24
    m, r = mean[:, None], rstd[:, None]
    xh = (x - m) * r
    exh = 2 * e * xh.abs() + e * r * (x.abs() + m.abs())
    w = dy * (1.0 if gamma is None else gamma)
    ew = e * w.abs()
    m1, m2 = w.mean(1, keepdim=True), (w * xh).mean(1, keepdim=True)
    em1 = (ew + depth * e * w.abs()).mean(1, keepdim=True)
    em2 = (w.abs() * exh + (depth + 2) * e * (w * xh).abs()).mean(1, keepdim=True)
    dx = r * (w - m1 - xh * m2)
    edx = r * (ew + em1 + exh * m2.abs() + xh.abs() * em2 + 4 * e * (w.abs() + m1.abs() + (xh * m2).abs()))
    dgamma, dbeta = (dy * xh).sum(0), dy.sum(0)
    edg = (dy.abs() * exh + deep * e * (dy * xh).abs()).sum(0)
    return {"dx": (dx, rounding(dx, edx, kind)), "dgamma": (dgamma, edg), "dbeta": (dbeta, deep * e * dy.abs().sum(0))}


def newton_schulz(g, steps, coefficients, eps, scale=1.0, rounded=lambda v: v):
    """The iteration in 64 bits on a batch [b, m, n]; `rounded` is applied wherever the operator stores a matrix."""
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    x = rounded(x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps))
    eye = torch.eye(x.shape[1], dtype=x.dtype, device=x.device)
    for s in range(steps):
        a, b, c = coefficients[s % len(coefficients)]
        p = rounded(x @ x.transpose(1, 2))
        q = rounded(a * eye + b * p + c * (p @ p))
        x = q @ x
        if s + 1 < steps:
            x = rounded(x)
    x = x * scale
    return (x.transpose(1, 2) if tall else x).contiguous()


def half_plane(v):
    """What one fp16 plane of 2^10 v holds."""
    return (v * 1024).to(torch.float16).to(v.dtype) / 1024


def check(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), "%s: not finite" % what
    off = (got - want).abs() - bound
    worst = off.max().item() if off.numel() else -1.0
    assert worst <= 0, "%s: %g over a bound of %g" % (what, worst, bound.flatten()[off.argmax()].item())
