"""The learner-side operators on the GPU against plain forms in 64 bits (tests/operator_bounds.py has the forms and the bounds)."""
import math

import pytest
import torch

import paper_2104_11125_b200 as sc
from paper_2104_11125_b200 import binding as b
from tests import operator_bounds as ob

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
KINDS = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["f32", "f16", "bf16"]
kinds = pytest.mark.parametrize("kind", KINDS, ids=IDS)


@pytest.fixture(scope="module")
def ops():
    with sc.Operators() as o:
        yield o
        assert o.status() == 0


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def spread(g, rows, cols, kind, pad=0, shift=0, scale=1.0):
    """A matrix whose rows are `pad` elements apart from one another and whose first element is `shift` elements off an
    allocation's start."""
    ld = cols + pad
    flat = torch.empty(shift + rows * ld + 8, device=DEV, dtype=kind)
    m = flat[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(randn(g, rows, cols) * scale)
    return m


def put(rows, cols, kind, pad=0, shift=0):
    """An output of the same layout filled with a marker, and a check that nothing around it was written."""
    ld = cols + pad
    flat = torch.full((shift + rows * ld + 8,), 7.0, device=DEV, dtype=kind)
    view = flat[shift:shift + rows * ld].view(rows, ld)

    def untouched():
        assert (flat[:shift] == 7.0).all() and (flat[shift + rows * ld:] == 7.0).all()
        assert (view[:, cols:] == 7.0).all()
    return view[:, :cols], untouched


# ---- layer norm ------------------------------------------------------------------------------------------------
LN_SHAPES = [(1, 1, 0, 0), (1, 512, 0, 0), (3, 2, 0, 0), (5, 31, 0, 1), (7, 33, 3, 0), (64, 128, 0, 0), (33, 257, 1, 3), (40, 1000, 8, 0),
             (9, 1024, 0, 0), (6, 1030, 0, 0), (5, 2047, 5, 0), (4, 4096, 0, 0), (3, 4104, 0, 8), (3, 8192, 0, 0), (2, 9000, 0, 0),
             (2, 16385, 0, 0), (600, 96, 0, 0), (1201, 64, 0, 0)]


@kinds
@pytest.mark.parametrize("rows,width,pad,shift", LN_SHAPES)
def test_layer_norm(ops, kind, rows, width, pad, shift):
    g = gen(rows * 131 + width)
    x = spread(g, rows, width, kind, pad, shift, 2.0)
    x += 0.5
    gamma, beta = 1 + 0.2 * randn(g, width), randn(g, width)
    for ga, be in ((gamma, beta), (None, beta), (gamma, None)):
        y, untouched = put(rows, width, kind, pad, shift)
        mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        ops.layer_norm(x, ga, be, 1e-5, y, mean, rstd)
        want = ob.layer_norm(x.double(), None if ga is None else ga.double(), None if be is None else be.double(), 1e-5, kind)
        ob.check(y, *want["y"], "y")
        ob.check(mean, *want["mean"], "mean")
        ob.check(rstd, *want["rstd"], "rstd")
        untouched()


@kinds
@pytest.mark.parametrize("rows,width,pad,shift", LN_SHAPES)
def test_layer_norm_backward(ops, kind, rows, width, pad, shift):
    g = gen(rows * 17 + width)
    x, dy = spread(g, rows, width, kind, pad, shift, 2.0), spread(g, rows, width, kind, 0, 0, 0.1)
    gamma = 1 + 0.2 * randn(g, width)
    xd = x.double()
    mean = xd.mean(1).float()
    rstd = (xd.var(1, correction=0) + 1e-5).rsqrt().float()
    for ga in (gamma, None):
        want = ob.layer_norm_backward(dy.double(), xd, None if ga is None else ga.double(), mean.double(), rstd.double(), kind)
        dx, untouched = put(rows, width, kind, pad, shift)
        dg, db = torch.full((width,), 7.0, device=DEV), torch.full((width,), 7.0, device=DEV)
        ops.layer_norm_backward(dy, x, ga, mean, rstd, dx, dg, db)
        ob.check(dx, *want["dx"], "dx")
        ob.check(dg, *want["dgamma"], "dgamma")
        ob.check(db, *want["dbeta"], "dbeta")
        untouched()
    # each output on its own, the same bits
    dx2 = torch.empty_like(dy)
    ops.layer_norm_backward(dy, x, None, mean, rstd, dx2)
    dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
    ops.layer_norm_backward(dy, x, None, mean, rstd, None, dg2, None)
    ops.layer_norm_backward(dy, x, None, mean, rstd, None, None, db2)
    ob.check(dx2, *want["dx"], "dx alone")
    ob.check(dg2, *want["dgamma"], "dgamma alone")
    ob.check(db2, *want["dbeta"], "dbeta alone")


@kinds
def test_layer_norm_in_place(ops, kind):
    g = gen(4)
    for rows, width in ((37, 200), (5, 20000)):
        x, dy = spread(g, rows, width, kind), spread(g, rows, width, kind)
        gamma = 1 + 0.1 * randn(g, width)
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        ops.layer_norm(x, gamma, None, 1e-5, y, mean, rstd)
        dx, dg, db = torch.empty_like(x), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
        ops.layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db)
        dy2, dg2, db2 = dy.clone(), torch.empty_like(dg), torch.empty_like(db)
        ops.layer_norm_backward(dy2, x, gamma, mean, rstd, dy2, dg2, db2)
        assert torch.equal(dy2, dx) and torch.equal(dg2, dg) and torch.equal(db2, db)
        x2 = x.clone()
        ops.layer_norm(x2, gamma, None, 1e-5, x2)
        assert torch.equal(x2, y)


@kinds
def test_layer_norm_special_rows(ops, kind):
    """Equal values, an offset much larger than the spread, NaN and infinities: each stays in its row."""
    g = gen(9)
    for width in (48, 700, 5000, 20000):
        x = spread(g, 8, width, kind)
        x[1] = 3.0
        x[2] = 0.0
        x[3, 5] = math.nan
        x[4, 7] = math.inf
        x[5, width - 1] = -math.inf
        gamma, beta = 1 + 0.1 * randn(g, width), randn(g, width)
        y, mean, rstd = torch.empty_like(x), torch.empty(8, device=DEV), torch.empty(8, device=DEV)
        ops.layer_norm(x, gamma, beta, 1e-5, y, mean, rstd)
        assert torch.equal(y[1], beta.to(kind)) and torch.equal(y[2], beta.to(kind))
        assert not torch.isfinite(y[3]).any() and not torch.isfinite(y[4]).any() and not torch.isfinite(y[5]).any()
        keep = [0, 6, 7]
        want = ob.layer_norm(x[keep].double(), gamma.double(), beta.double(), 1e-5, kind)
        ob.check(y[keep], *want["y"], "rows beside")
    # mean 1000 times the spread: the differences are what counts (values chosen so that they are exact in the type)
    step = 8.0 if kind == torch.bfloat16 else 1.0
    x = (1024 + step * torch.randint(0, 4, (6, 640), generator=g, device=DEV)).to(kind)
    y = torch.empty_like(x)
    ops.layer_norm(x, None, None, 0.0, y)
    want = ob.layer_norm(x.double(), None, None, 0.0, kind)
    ob.check(y, *want["y"], "offset rows")


def test_layer_norm_long_buffers(ops):
    """Offsets beyond 2^31 elements."""
    rows, width = (1 << 20) + 3, 2304
    x = torch.zeros(rows, width, device=DEV, dtype=torch.bfloat16)
    g = gen(12)
    x[-4:] = randn(g, 4, width).to(torch.bfloat16)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ops.layer_norm(x, None, None, 1e-5, y, mean, rstd)
    want = ob.layer_norm(x[-4:].double(), None, None, 1e-5, torch.bfloat16)
    ob.check(y[-4:], *want["y"], "last rows")
    assert (y[:-4] == 0).all()
    dx, dg, db = torch.empty_like(x), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
    ops.layer_norm_backward(x, x, None, mean, rstd, dx, dg, db)
    back = ob.layer_norm_backward(x[-4:].double(), x[-4:].double(), None, mean[-4:].double(), rstd[-4:].double(), torch.bfloat16)
    ob.check(dx[-4:], *back["dx"], "last rows' dx")
    ob.check(dg, *back["dgamma"], "dgamma")


def test_layer_norm_gradient_against_differences(ops):
    g = gen(21)
    rows, width = 11, 77
    x, dy, v = randn(g, rows, width), randn(g, rows, width), randn(g, rows, width)
    gamma, beta = 1 + 0.2 * randn(g, width), randn(g, width)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ops.layer_norm(x, gamma, beta, 1e-5, y, mean, rstd)
    dx, dg, db = torch.empty_like(x), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
    ops.layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db)

    def loss(a, ga, be):
        out = torch.empty_like(a)
        ops.layer_norm(a, ga, be, 1e-5, out)
        return (out.double() * dy.double()).sum().item()
    # central differences: h^2 of a third derivative of order |v|^3 / width, and 2^-22 |y| |dy| / h of rounding
    h = 2.0 ** -7
    size = (y.double().norm() * dy.double().norm()).item()
    tol = 2.0 ** -22 * size / h + 4 * h * h * size
    vg, vb = randn(g, width), randn(g, width)
    assert abs((loss(x + h * v, gamma, beta) - loss(x - h * v, gamma, beta)) / (2 * h) - (dx.double() * v.double()).sum().item()) < tol
    assert abs((loss(x, gamma + h * vg, beta) - loss(x, gamma - h * vg, beta)) / (2 * h) - (dg.double() * vg.double()).sum().item()) < tol
    assert abs((loss(x, gamma, beta + h * vb) - loss(x, gamma, beta - h * vb)) / (2 * h) - (db.double() * vb.double()).sum().item()) < tol


# ---- gated feed-forward --------------------------------------------------------------------------------------------
def ffn_inputs(seed, t, d, f, kind, pad=0, shift=0):
    g = gen(seed)
    x = spread(g, t, d, kind, pad, shift)
    wg, wu = (randn(g, f, d) / math.sqrt(d)).to(kind), (randn(g, f, d) / math.sqrt(d)).to(kind)
    wd = (randn(g, d, f) / math.sqrt(f)).to(kind)
    dy = spread(g, t, d, kind, pad, shift, 0.25)
    return x, wg, wu, wd, dy


FFN_SHAPES = [(1, 1, 1, 0, 0), (1, 64, 128, 0, 0), (1, 257, 131, 0, 0), (2, 96, 72, 0, 0), (3, 130, 65, 2, 1), (5, 8, 1000, 0, 0), (8, 512, 512, 0, 0),
              (17, 24, 40, 8, 0), (64, 136, 264, 0, 0), (127, 65, 129, 1, 0), (128, 64, 128, 0, 0), (129, 192, 320, 0, 0), (200, 1001, 300, 3, 5),
              (300, 72, 1030, 0, 0), (520, 264, 392, 0, 8), (1000, 40, 24, 0, 0)]


@kinds
@pytest.mark.parametrize("t,d,f,pad,shift", FFN_SHAPES)
@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_ffn(ops, kind, t, d, f, pad, shift, name):
    x, wg, wu, wd, _ = ffn_inputs(t + d + f, t, d, f, kind, pad, shift)
    want = ob.ffn(x.double(), wg.double(), wu.double(), wd.double(), name, kind)
    y, untouched = put(t, d, kind, pad, shift)
    ops.gated_ffn(x, wg, wu, wd, y, activation=name)
    ob.check(y, *want["y"], "y")
    untouched()
    saved, y2 = torch.empty(2, t, f, device=DEV, dtype=kind), torch.empty(t, d, device=DEV, dtype=kind)
    ops.gated_ffn(x, wg, wu, wd, y2, saved=saved, activation=name)
    ob.check(y2, *want["y"], "y beside saved")
    ob.check(saved, *want["saved"], "saved")


@kinds
@pytest.mark.parametrize("t,d,f,pad,shift", FFN_SHAPES)
@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_ffn_backward(ops, kind, t, d, f, pad, shift, name):
    x, wg, wu, wd, dy = ffn_inputs(t * 3 + d + f, t, d, f, kind, pad, shift)
    y, saved = torch.empty(t, d, device=DEV, dtype=kind), torch.empty(2, t, f, device=DEV, dtype=kind)
    ops.gated_ffn(x, wg, wu, wd, y, saved=saved, activation=name)
    for wgrad in {kind, torch.float32}:
        want = ob.ffn(x.double(), wg.double(), wu.double(), wd.double(), name, kind, dy.double(), wgrad)
        dx, untouched = put(t, d, kind, pad, shift)
        dwg, dwu = torch.empty(f, d, device=DEV, dtype=wgrad), torch.empty(f, d, device=DEV, dtype=wgrad)
        dwd = torch.empty(d, f, device=DEV, dtype=wgrad)
        ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, dx, dwg, dwu, dwd, activation=name)
        for key, got in (("dx", dx), ("dw_gate", dwg), ("dw_up", dwu), ("dw_down", dwd)):
            ob.check(got, *want[key], key)
        untouched()
        # any of them alone
        alone = torch.empty_like(dwu)
        ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, None, None, alone, None, activation=name)
        assert torch.equal(alone, dwu)
        alone = torch.empty_like(dwd)
        ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, None, None, None, alone, activation=name)
        assert torch.equal(alone, dwd)


@kinds
def test_gated_ffn_gradients_in_a_flat_vector(ops, kind):
    """Weight gradients as slices of one learner's fp32 gradient vector, at offsets that are no multiple of 16 bytes."""
    t, d, f = 70, 45, 83
    x, wg, wu, wd, dy = ffn_inputs(5, t, d, f, kind)
    y, saved = torch.empty(t, d, device=DEV, dtype=kind), torch.empty(2, t, f, device=DEV, dtype=kind)
    ops.gated_ffn(x, wg, wu, wd, y, saved=saved)
    flat = torch.full((3 * d * f + 5,), 7.0, device=DEV)
    parts = [flat[1 + i * d * f:1 + (i + 1) * d * f] for i in range(3)]
    dx = torch.empty_like(dy)
    ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, dx, parts[0].view(f, d), parts[1].view(f, d), parts[2].view(d, f))
    want = ob.ffn(x.double(), wg.double(), wu.double(), wd.double(), "silu", kind, dy.double(), torch.float32)
    for key, p, s in (("dw_gate", parts[0], (f, d)), ("dw_up", parts[1], (f, d)), ("dw_down", parts[2], (d, f))):
        ob.check(p.view(*s), *want[key], key)
    assert flat[0] == 7.0 and (flat[-4:] == 7.0).all()


def test_gated_ffn_larger_sizes(ops):
    """Several tiles a block, parts of k joined, wide and narrow tiles."""
    for kind, t, d, f, name in ((torch.bfloat16, 2000, 520, 2056, "silu"), (torch.float16, 700, 1024, 4096, "gelu"), (torch.float32, 515, 768, 1500, "silu"),
                                (torch.bfloat16, 24, 2048, 4096, "silu"), (torch.bfloat16, 4096, 64, 96, "relu")):
        x, wg, wu, wd, dy = ffn_inputs(t, t, d, f, kind)
        want = ob.ffn(x.double(), wg.double(), wu.double(), wd.double(), name, kind, dy.double(), torch.float32)
        y, saved = torch.empty(t, d, device=DEV, dtype=kind), torch.empty(2, t, f, device=DEV, dtype=kind)
        ops.gated_ffn(x, wg, wu, wd, y, saved=saved, activation=name)
        dx = torch.empty_like(x)
        dwg, dwu, dwd = torch.empty(f, d, device=DEV), torch.empty(f, d, device=DEV), torch.empty(d, f, device=DEV)
        ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, dx, dwg, dwu, dwd, activation=name)
        for key, got in (("y", y), ("saved", saved), ("dx", dx), ("dw_gate", dwg), ("dw_up", dwu), ("dw_down", dwd)):
            ob.check(got, *want[key], "%s %s" % (kind, key))


def test_gated_ffn_long_buffers(ops):
    """tokens * hidden beyond 2^31."""
    t, d, f = (1 << 18) + 1, 64, 8704
    x, wg, wu, wd, _ = ffn_inputs(1, 4, d, f, torch.bfloat16)
    long = torch.zeros(t, d, device=DEV, dtype=torch.bfloat16)
    long[-4:] = x
    y, saved = torch.empty_like(long), torch.empty(2, t, f, device=DEV, dtype=torch.bfloat16)
    ops.gated_ffn(long, wg, wu, wd, y, saved=saved)
    want = ob.ffn(x.double(), wg.double(), wu.double(), wd.double(), "silu", torch.bfloat16)
    ob.check(y[-4:], *want["y"], "last rows")
    ob.check(saved[:, -4:], *want["saved"], "last rows' saved")
    assert (y[:-4] == 0).all()


@kinds
def test_gated_ffn_keeps_rows_apart(ops, kind):
    """A NaN in one token reaches that token's row only; very different magnitudes stand side by side."""
    for t in (3, 40, 150):
        x, wg, wu, wd, _ = ffn_inputs(8, t, 96, 160, kind)
        y0, y1 = torch.empty(t, 96, device=DEV, dtype=kind), torch.empty(t, 96, device=DEV, dtype=kind)
        ops.gated_ffn(x, wg, wu, wd, y0)
        x2 = x.clone()
        x2[1, 5] = math.nan
        ops.gated_ffn(x2, wg, wu, wd, y1)
        keep = [i for i in range(t) if i != 1]
        assert not torch.isfinite(y1[1]).any()
        assert torch.equal(y1[keep], y0[keep])
    if kind == torch.float32:
        x = randn(gen(2), 6, 96)
        x[2] *= 2.0 ** 12
        x[4] *= 2.0 ** -6
        y = torch.empty_like(x)
        ops.gated_ffn(x, wg, wu, wd, y, activation="relu")
        want = ob.ffn(x.double(), wg.double(), wu.double(), wd.double(), "relu", kind)
        ob.check(y, *want["y"], "rows of different size")


def test_gated_ffn_scaled_by_powers_of_two(ops):
    """fp32 operands far from one: relu's block is homogeneous, so a power of two goes through exactly."""
    x, wg, wu, wd, dy = ffn_inputs(3, 50, 40, 56, torch.float32)
    outs = []
    for e in (0, -40, 30):
        s = 2.0 ** e
        y, saved = torch.empty_like(x), torch.empty(2, 50, 56, device=DEV)
        ops.gated_ffn(x * s, wg, wu, wd, y, saved=saved, activation="relu")
        dx, dw = torch.empty_like(x), torch.empty_like(wd)
        ops.gated_ffn_backward(dy * s, x * s, wg, wu, wd, saved, dx, None, None, dw, activation="relu")
        outs.append((y / s / s, dx / s / s, dw / s / s / s))
    for o in outs[1:]:
        for p, q in zip(o, outs[0]):
            assert torch.equal(p, q)


def test_gated_ffn_gradient_against_differences(ops):
    t, d, f = 6, 40, 56
    x, wg, wu, wd, dy = ffn_inputs(77, t, d, f, torch.float32)
    g = gen(78)
    saved, y = torch.empty(2, t, f, device=DEV), torch.empty_like(x)
    ops.gated_ffn(x, wg, wu, wd, y, saved=saved)
    grads = [torch.empty_like(v) for v in (x, wg, wu, wd)]
    ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, *grads)

    def loss(*args):
        out = torch.empty_like(x)
        ops.gated_ffn(*args, out)
        return (out.double() * dy.double()).sum().item()
    h = 2.0 ** -7
    for i in range(4):
        args = [x, wg, wu, wd]
        v = randn(g, *args[i].shape) * (1.0 if i == 0 else 0.1)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * v, args[i] - h * v
        got = (loss(*up) - loss(*down)) / (2 * h)
        # rounding of a forward pass (2^-19 of the sizes multiplied) over h, and the cubic term of the differences
        size = (y.double().norm() * dy.double().norm()).item()
        tol = 2.0 ** -19 * size / h + 16 * h * h * size
        assert abs(got - (grads[i].double() * v.double()).sum().item()) < tol


# ---- Newton-Schulz -------------------------------------------------------------------------------------------------
CO = [(3.4445, -4.7750, 2.0315)]
NS_SHAPES = [(1, 1, 1), (2, 1, 9), (2, 9, 1), (1, 16, 16), (3, 17, 40), (2, 40, 17), (1, 64, 256), (2, 100, 90), (1, 127, 129), (2, 128, 128),
             (1, 130, 300), (1, 300, 130), (1, 257, 257), (2, 384, 1000), (1, 1000, 392)]


def ns_close(got, g, steps, co, scale, out_kind):
    """The operator's distance from the iteration in 64 bits, against what the iteration loses when every stored matrix is
    rounded as the operator rounds it (one fp16 plane; for fp32 two, taken as a relative perturbation of 2^-22 and 2^-20 for
    the sums).  Twice that, for another pattern of the same roundings, and the output's own rounding."""
    exact = ob.newton_schulz(g, steps, co, 1e-7, scale)
    if out_kind == torch.float32:
        r = gen(1)

        def rounded(v):
            noise = torch.randn(v.shape, generator=r, device=DEV, dtype=torch.float64)
            return v + 2.0 ** -20 * noise * v.abs() + 2.0 ** -35 * noise
    else:
        rounded = ob.half_plane
    model = ob.newton_schulz(g, steps, co, 1e-7, scale, rounded)
    norm = exact.flatten(1).norm(dim=1)
    tol = 2 * (model - exact).flatten(1).norm(dim=1) + 2 * ob.U[out_kind] * norm + 2.0 ** -24 * abs(scale)
    off = (got.double() - exact).flatten(1).norm(dim=1)
    assert torch.isfinite(got).all()
    assert (off <= tol).all(), (off / norm, tol / norm)


@kinds
@pytest.mark.parametrize("batch,rows,cols", NS_SHAPES)
def test_orthogonalise(ops, kind, batch, rows, cols):
    g = randn(gen(rows * cols), batch, rows, cols) * 1e-3
    out = torch.empty(batch, rows, cols, device=DEV, dtype=kind)
    ops.orthogonalise(g, out)
    ns_close(out, g.double(), 5, CO, 1.0, kind)
    if kind != torch.float32:                                     # inputs of the output's type, in place
        h = g.to(kind)
        want = h.double()
        ops.orthogonalise(h, h, scale=-0.5)
        ns_close(h, want, 5, CO, -0.5, kind)


@kinds
def test_orthogonalise_layouts(ops, kind):
    """Slices of a flat vector at odd offsets, rows apart, one matrix without a batch dimension, a coefficient triple a step."""
    co = [(4.0, -6.0, 3.0), (3.0, -3.2, 1.2), (1.875, -1.25, 0.375)]
    r = gen(31)
    flat = randn(r, 7 * 3 * 50 * 33)
    upd = flat[3:3 + 3 * 50 * 40].view(3, 50, 40)[:, :, :33]
    buf = torch.full((5 + 3 * 50 * 37,), 7.0, device=DEV, dtype=kind)
    out = buf[5:].view(3, 50, 37)[:, :, :33]
    ops.orthogonalise(upd, out, steps=3, coefficients=co)
    ns_close(out.contiguous(), upd.double().contiguous(), 3, co, 1.0, kind)
    assert (buf[:5] == 7.0).all() and (buf[5:].view(3, 50, 37)[:, :, 33:] == 7.0).all()
    one = torch.empty(50, 33, device=DEV, dtype=kind)
    ops.orthogonalise(upd[1], one, steps=3, coefficients=co)
    assert torch.equal(one, out[1])
    ops.orthogonalise(upd[1], one, steps=0, coefficients=(1.0, 0.0, 0.0), scale=3.0)
    want = 3 * upd[1].double() / (upd[1].double().norm() + 1e-7)
    ob.check(one, want, ob.rounding(want, 2.0 ** -22 * want.abs(), kind), "no steps")


@kinds
def test_orthogonalise_extremes(ops, kind):
    """A zero matrix, magnitudes near both ends of fp32, a NaN in one matrix of a batch, a matrix of rank one."""
    r = gen(41)
    for rows, cols in ((24, 40), (140, 200)):
        g = randn(r, 5, rows, cols)
        g[1] = 0
        g[2, 3, 4] = math.nan
        g[4] = randn(r, rows, 1) @ randn(r, 1, cols)
        out = torch.empty(5, rows, cols, device=DEV, dtype=kind)
        ops.orthogonalise(g, out)
        assert (out[1] == 0).all()
        assert torch.isnan(out[2]).all()
        keep = [0, 3, 4]
        ns_close(out[keep], g[keep].double(), 5, CO, 1.0, kind)
        for e in (-60, 100):
            o2 = torch.empty(2, rows, cols, device=DEV, dtype=kind)
            ops.orthogonalise(g[keep[:2]] * 2.0 ** e, o2, eps=0.0)
            o3 = torch.empty(2, rows, cols, device=DEV, dtype=kind)
            ops.orthogonalise(g[keep[:2]].contiguous(), o3, eps=0.0)
            assert torch.equal(o2, o3)


def test_orthogonalise_larger_sizes(ops):
    for batch, rows, cols, kind in ((3, 512, 2048, torch.bfloat16), (1, 1024, 1024, torch.float16), (2, 700, 515, torch.float32), (1, 2050, 640, torch.bfloat16)):
        g = randn(gen(rows), batch, rows, cols)
        out = torch.empty(batch, rows, cols, device=DEV, dtype=kind)
        ops.orthogonalise(g, out)
        ns_close(out, g.double(), 5, CO, 1.0, kind)


# ---- all of them: determinism, streams, handles, refusals ---------------------------------------------------------------
@kinds
def test_calls_repeat_bit_for_bit_and_share_scratch(ops, kind):
    def run(o):
        res = []
        for t, d, f in ((300, 200, 410), (1, 64, 80), (90, 520, 1030)):
            x, wg, wu, wd, dy = ffn_inputs(t, t, d, f, kind)
            y, saved = torch.empty_like(x), torch.empty(2, t, f, device=DEV, dtype=kind)
            o.gated_ffn(x, wg, wu, wd, y, saved=saved)
            grads = [torch.empty_like(v) for v in (x, wg, wu, wd)]
            o.gated_ffn_backward(dy, x, wg, wu, wd, saved, *grads)
            mean, rstd = x.float().mean(1), x.float().var(1, correction=0).add(1e-5).rsqrt()
            dx, dg, db = torch.empty_like(x), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
            o.layer_norm_backward(dy, x, None, mean, rstd, dx, dg, db)
            q = torch.empty_like(wg)
            o.orthogonalise(wg, q)
            res += [y, *grads, dx, dg, db, q]
        return res
    a, c = run(ops), run(ops)
    with sc.Operators() as fresh:                     # scratch that grows from nothing on the way
        e = run(fresh)
        assert fresh.status() == 0 and fresh.workspace() > 0
    for p, q, r in zip(a, c, e):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_on_another_stream(ops):
    s = torch.cuda.Stream()
    x, wg, wu, wd, dy = ffn_inputs(2, 200, 256, 512, torch.bfloat16)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    ops.gated_ffn(x, wg, wu, wd, y0)
    torch.cuda.synchronize()
    with sc.Operators(stream=s) as o:
        o.reserve(64 << 20)
        assert o.workspace() >= 64 << 20
        with torch.cuda.stream(s):
            x2 = torch.empty_like(x)
            torch.cuda._sleep(20_000_000)             # the copy below is late; the call has to come after it
            x2.copy_(x)
            o.gated_ffn(x2, wg, wu, wd, y1)
        s.synchronize()
        assert torch.equal(y0, y1)
        o.set_stream(None)
        assert o.status() == 0


def test_in_a_cuda_graph(ops):
    s = torch.cuda.Stream()
    x, wg, wu, wd, dy = ffn_inputs(6, 64, 128, 256, torch.float32)
    with sc.Operators(stream=s) as o:
        y, saved, q = torch.empty_like(x), torch.empty(2, 64, 256, device=DEV), torch.empty_like(wg)
        grads = [torch.empty_like(v) for v in (x, wg, wu, wd)]

        def work():
            o.gated_ffn(x, wg, wu, wd, y, saved=saved)
            o.gated_ffn_backward(dy, x, wg, wu, wd, saved, *grads)
            o.orthogonalise(grads[1], q)
        torch.cuda.synchronize()
        work()                                        # scratch is allocated before the capture
        s.synchronize()
        want = [v.clone() for v in (y, *grads, q)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        for v in (y, *grads, q):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for v, w in zip((y, *grads, q), want):
            assert torch.equal(v, w)


def test_sizes_of_zero(ops):
    L, h = sc.operators.lib(), ops._h
    w = torch.full((3, 4), 7.0, device=DEV)
    p = w.data_ptr()
    assert L.scalecom_layer_norm(h, 0, 0, 4, None, 4, None, None, 1e-5, None, 4, None, None) == 0
    dg, db = torch.full((4,), 7.0, device=DEV), torch.full((4,), 7.0, device=DEV)
    assert L.scalecom_layer_norm_backward(h, 0, 0, 4, None, 4, None, 4, None, None, None, None, 4, dg.data_ptr(), db.data_ptr()) == 0
    assert (dg == 0).all() and (db == 0).all()
    assert L.scalecom_gated_ffn(h, 0, 0, 0, 4, 3, None, 4, p, p, p, None, 4, None) == 0
    assert L.scalecom_gated_ffn_backward(h, 0, 0, 0, 0, 4, 3, None, 4, None, 4, None, None, None, None, None, 4, p, None, None) == 0
    torch.cuda.synchronize()
    assert (w == 0).all()
    assert L.scalecom_orthogonalise(h, 0, 4, 3, 0, None, 3, 12, 0, None, 3, 12, 0, None, 1, 0.0, 1.0) == 0


def test_refusals(ops):
    """Every bad argument is an error code, and nothing has been written."""
    L, h = sc.operators.lib(), ops._h
    bufs = [torch.full((64, 64), 7.0, device=DEV) for _ in range(12)]
    a, c, d, e, f, g, k, m, n, q, r, s = [t.data_ptr() for t in bufs]
    big, nan, inf = (1 << 26) + 1, math.nan, math.inf

    def ln(dt=0, rows=8, width=8, x=a, ldx=8, gamma=None, beta=None, eps=1e-5, y=c, ldy=8, mean=None, rstd=None, hh=h):
        return L.scalecom_layer_norm(hh, dt, rows, width, x, ldx, gamma, beta, eps, y, ldy, mean, rstd)
    for kw in (dict(dt=3), dict(dt=-1), dict(rows=-1), dict(rows=big), dict(width=0), dict(width=big), dict(ldx=7), dict(ldy=7),
               dict(eps=-1.0), dict(eps=nan), dict(eps=inf)):
        assert ln(**kw) == b.ERR_INVALID_ARG, kw
    for kw in (dict(x=None), dict(y=None)):
        assert ln(**kw) == b.ERR_NULL_PTR, kw
    for kw in (dict(y=a, ldy=9), dict(gamma=c), dict(beta=c), dict(mean=c), dict(rstd=c), dict(mean=d, rstd=d), dict(mean=a), dict(rstd=a)):
        assert ln(**kw) == b.ERR_ALIAS, kw

    def lb(dt=0, rows=8, width=8, dy=a, lddy=8, x=c, ldx=8, gamma=d, mean=e, rstd=f, dx=g, lddx=8, dgamma=k, dbeta=m):
        return L.scalecom_layer_norm_backward(h, dt, rows, width, dy, lddy, x, ldx, gamma, mean, rstd, dx, lddx, dgamma, dbeta)
    for kw in (dict(dt=7), dict(rows=-2), dict(width=0), dict(ldx=1), dict(lddy=1), dict(lddx=1)):
        assert lb(**kw) == b.ERR_INVALID_ARG, kw
    for kw in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None)):
        assert lb(**kw) == b.ERR_NULL_PTR, kw
    for kw in (dict(dx=c), dict(dx=a, lddx=9), dict(dx=d), dict(dx=e), dict(dx=f), dict(dgamma=m), dict(dgamma=a), dict(dbeta=c), dict(dgamma=d),
               dict(dbeta=f), dict(dx=k)):
        assert lb(**kw) == b.ERR_ALIAS, kw

    def ff(dt=0, act=0, t=8, w=8, hid=8, x=a, ldx=8, wg=c, wu=d, wd=e, y=f, ldy=8, saved=g):
        return L.scalecom_gated_ffn(h, dt, act, t, w, hid, x, ldx, wg, wu, wd, y, ldy, saved)
    for kw in (dict(dt=3), dict(act=4), dict(act=-1), dict(t=-1), dict(t=big), dict(w=0), dict(hid=0), dict(hid=big), dict(ldx=7), dict(ldy=7)):
        assert ff(**kw) == b.ERR_INVALID_ARG, kw
    for kw in (dict(x=None), dict(wg=None), dict(wu=None), dict(wd=None), dict(y=None)):
        assert ff(**kw) == b.ERR_NULL_PTR, kw
    for kw in (dict(y=a), dict(y=c), dict(y=e), dict(saved=a), dict(saved=f), dict(saved=d)):
        assert ff(**kw) == b.ERR_ALIAS, kw

    def fb(dt=0, wt=0, act=0, t=8, w=8, hid=8, dy=a, lddy=8, x=c, ldx=8, wg=d, wu=e, wd=f, saved=g, dx=k, lddx=8, dwg=m, dwu=n, dwd=q):
        return L.scalecom_gated_ffn_backward(h, dt, wt, act, t, w, hid, dy, lddy, x, ldx, wg, wu, wd, saved, dx, lddx, dwg, dwu, dwd)
    for kw in (dict(dt=3), dict(wt=1), dict(dt=1, wt=2), dict(act=9), dict(t=-1), dict(w=0), dict(hid=0), dict(ldx=7), dict(lddy=7), dict(lddx=7)):
        assert fb(**kw) == b.ERR_INVALID_ARG, kw
    for kw in (dict(dy=None), dict(x=None), dict(wg=None), dict(wu=None), dict(wd=None), dict(saved=None)):
        assert fb(**kw) == b.ERR_NULL_PTR, kw
    for kw in (dict(dx=a), dict(dx=m), dict(dwg=n), dict(dwd=g), dict(dwu=e), dict(dx=c)):
        assert fb(**kw) == b.ERR_ALIAS, kw

    import ctypes
    co = (ctypes.c_float * 3)(3.4, -4.7, 2.0)
    bad = (ctypes.c_float * 3)(64.0, -4.7, 2.0)
    worse = (ctypes.c_float * 3)(3.4, nan, 2.0)
    cp = [ctypes.cast(v, ctypes.c_void_p) for v in (co, bad, worse)]

    def ns(batch=2, rows=8, cols=8, it=0, x=a, ldi=8, si=64, ot=0, y=c, ldo=8, so=64, steps=5, coef=cp[0], nc=1, eps=1e-7, scale=1.0):
        return L.scalecom_orthogonalise(h, batch, rows, cols, it, x, ldi, si, ot, y, ldo, so, steps, coef, nc, eps, scale)
    for kw in (dict(batch=-1), dict(batch=70000), dict(rows=0), dict(cols=0), dict(cols=big), dict(it=5), dict(ot=-1), dict(ldi=7), dict(ldo=7), dict(si=63),
               dict(so=10), dict(steps=-1), dict(steps=65), dict(nc=2), dict(nc=0), dict(coef=cp[1]), dict(coef=cp[2]), dict(eps=-1.0), dict(eps=nan),
               dict(scale=inf)):
        assert ns(**kw) == b.ERR_INVALID_ARG, kw
    for kw in (dict(x=None), dict(y=None), dict(coef=None)):
        assert ns(**kw) == b.ERR_NULL_PTR, kw
    for kw in (dict(y=a, ldo=9, so=72), dict(y=a, ot=1), dict(y=a, so=128)):
        assert ns(**kw) == b.ERR_ALIAS, kw
    assert L.scalecom_ops_reserve(h, -1) == b.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in bufs)
    assert ops.status() == 0


def test_the_binding_checks_tensors(ops):
    x = torch.zeros(4, 8, device=DEV)
    w = torch.zeros(6, 8, device=DEV)
    wd = torch.zeros(8, 6, device=DEV)
    with pytest.raises(TypeError):
        ops.layer_norm(x.double(), None, None, 1e-5, x.double())
    with pytest.raises(TypeError):
        ops.layer_norm(x, None, None, 1e-5, x.half())
    with pytest.raises(ValueError):
        ops.layer_norm(x, None, None, 1e-5, torch.zeros(4, 9, device=DEV))
    with pytest.raises(ValueError):
        ops.layer_norm(torch.zeros(8, 4, device=DEV).t(), None, None, 1e-5, x)
    with pytest.raises(TypeError):
        ops.layer_norm(x, torch.zeros(7, device=DEV), None, 1e-5, torch.empty_like(x))
    with pytest.raises(ValueError):
        ops.gated_ffn(x, w, w, w, torch.empty_like(x))
    with pytest.raises(TypeError):
        ops.gated_ffn(x, w.half(), w, wd, torch.empty_like(x))
    with pytest.raises(KeyError):
        ops.gated_ffn(x, w, w, wd, torch.empty_like(x), activation="tanh")
    with pytest.raises(ValueError):
        ops.gated_ffn(x, w, w, wd, torch.empty_like(x), saved=torch.zeros(2, 4, 7, device=DEV))
    with pytest.raises(TypeError):
        ops.gated_ffn_backward(x, x, w, w, wd, torch.zeros(2, 4, 6, device=DEV), torch.empty_like(x), w.half())
    with pytest.raises(ValueError):
        ops.orthogonalise(w, torch.empty_like(w), steps=3, coefficients=[(1.0, 0.0, 0.0)] * 2)
    with pytest.raises(sc.ScaleComError) as err:
        ops.orthogonalise(w, torch.empty_like(w), coefficients=(100.0, 0.0, 0.0))
    assert err.value.code == b.ERR_INVALID_ARG
