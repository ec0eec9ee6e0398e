"""The learner-side operators where one of their parts meets another: launches of several products, values at the edges of what a
type or a scale holds, arguments that share memory."""
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


# ---- gated feed-forward block ------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", KINDS[1:], ids=IDS[1:])
@pytest.mark.parametrize("t,d,f", [(8192, 1024, 128), (16384, 512, 128), (16384, 520, 72)])
def test_outputs_of_both_sizes_in_one_launch(ops, kind, t, d, f):
    """16-bit activations with fp32 weight gradients and more tokens than twice the hidden size: the gradients' products, whose
    sums over the tokens are the longest, come before dx in one launch, so the same warps store blocks of 32 bits and then of 16.
    The launch with 16-bit gradients sums in the same order and stores blocks of one size: dx has to be the same bits, and its
    gradients the fp32 ones rounded."""
    g = gen(t + d)
    x, dy = randn(g, t, d).to(kind), (0.25 * randn(g, t, d)).to(kind)
    wg, wu = (randn(g, f, d) / math.sqrt(d)).to(kind), (randn(g, f, d) / math.sqrt(d)).to(kind)
    wd = (randn(g, d, f) / math.sqrt(f)).to(kind)
    y, saved = torch.empty_like(x), torch.empty(2, t, f, device=DEV, dtype=kind)
    ops.gated_ffn(x, wg, wu, wd, y, saved=saved)

    def grads(wide):
        out = [torch.empty_like(x)] + [torch.empty(w.shape, device=DEV, dtype=torch.float32 if wide else kind) for w in (wg, wu, wd)]
        ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, *out)
        return out
    narrow = grads(False)
    first = grads(True)
    for again in range(20):
        wide = first if not again else grads(True)
        assert torch.equal(wide[0], narrow[0])
        for p, q, r in zip(wide[1:], narrow[1:], first[1:]):
            assert torch.equal(p.to(kind), q) and torch.equal(p, r)


@pytest.mark.parametrize("ex,ew", [(64, 58), (-60, -62), (-2, 70), (-70, 10)])
def test_fp32_products_of_far_scales(ops, ex, ew):
    """Operands whose scales multiply to more, or less, than a fp32 holds, and whose products it holds: sums of 8 powers of two are
    exact. Rows and columns whose products pass the type's range stand beside them and are left out."""
    t, d, f = 40, 8, 24
    x = torch.full((t, d), 2.0 ** ex, device=DEV)
    wg, wu, wd = torch.full((f, d), 2.0 ** ew, device=DEV), torch.full((f, d), 2.0 ** ew, device=DEV), torch.ones(d, f, device=DEV)
    if ex > 0:
        x[0] *= 2.0 ** 36
        wg[1:] *= 2.0 ** -20
    y, saved = torch.empty_like(x), torch.empty(2, t, f, device=DEV)
    ops.gated_ffn(x, wg, wu, wd, y, saved=saved, activation="relu")
    for got, w in ((saved[0], wg), (saved[1], wu)):
        want = x.double() @ w.double().t()
        keep = want < 2.0 ** 128
        assert keep[1:, 1:].all() and torch.equal(got.double()[keep], want[keep])


def test_fp32_gradients_of_far_scales(ops):
    """dw_down = dy^T h with both around 2^-62: every sum is an exact power of two far above the smallest fp32."""
    t, d, f = 32, 8, 24
    x, wg = torch.full((t, d), 2.0 ** -20, device=DEV), torch.full((f, d), 2.0 ** -11, device=DEV)
    dy, saved = torch.full((t, d), 2.0 ** -68, device=DEV), torch.full((2, t, f), 2.0 ** -28, device=DEV)
    dwd = torch.empty(d, f, device=DEV)
    ops.gated_ffn_backward(dy, x, wg, wg.clone(), torch.ones(d, f, device=DEV), saved, None, None, None, dwd, activation="relu")
    assert (dwd.double() == t * 2.0 ** -124).all()


@pytest.mark.parametrize("t,d,f", [(50, 40, 56), (300, 136, 264), (1000, 520, 1030)])
@pytest.mark.parametrize("name,which", [("silu", "w_up"), ("gelu", "w_up"), ("relu", "w_up"), ("relu", "w_gate")])
def test_fp32_weights_of_far_sizes(ops, t, d, f, name, which):
    """The block is linear in w_up, and relu's homogeneous in w_gate: 2^-30 of either goes through all of it exactly. Each tensor keeps its
    bits whatever its neighbour's size."""
    g = gen(t + d)
    x, dy = randn(g, t, d), 0.25 * randn(g, t, d)
    wg, wu, wd = randn(g, f, d) / math.sqrt(d), randn(g, f, d) / math.sqrt(d), randn(g, d, f) / math.sqrt(f)
    s = 2.0 ** -30
    runs = []
    for a in (1.0, s):
        wg2, wu2 = (wg, wu * a) if which == "w_up" else (wg * a, wu)
        y, saved, grads = torch.empty_like(x), torch.empty(2, t, f, device=DEV), [torch.empty_like(v) for v in (x, wg, wu, wd)]
        ops.gated_ffn(x, wg2, wu2, wd, y, saved=saved, activation=name)
        ops.gated_ffn_backward(dy, x, wg2, wu2, wd, saved, *grads, activation=name)
        runs.append([y, saved[0], saved[1], *grads])
    # y, g, u, dx, dw_gate, dw_up, dw_down; the gradient of the weights that shrank stays
    small = (1, 0, 1, 1, 1, 0, 1) if which == "w_up" else (1, 1, 0, 1, 0, 1, 1)
    for p, q, scaled in zip(*runs, small):
        assert torch.equal(q, p * s if scaled else p)


# ---- layer norm ------------------------------------------------------------------------------------------------
@kinds
@pytest.mark.parametrize("width", [1, 2, 7, 13, 26, 49, 96, 128, 255, 300, 1001, 1024, 2047, 2048, 4096, 5000, 8192, 9000])
@pytest.mark.parametrize("shift", [0, 1])
def test_rows_of_equal_values_give_beta(ops, kind, width, shift):
    """Of any width, on the 16-byte grid and off it: the mean is the value itself, and 1 / sqrt(eps) has nothing to magnify."""
    values = torch.tensor([1.0, 3.0, 1000.0, 1000.1, -0.3, 7e-6, 6.1e4, 0.0], device=DEV).to(kind)
    rows = len(values)
    flat = torch.empty(shift + rows * width, device=DEV, dtype=kind)
    x = flat[shift:].view(rows, width)
    x.copy_(values[:, None].expand(rows, width))
    g = gen(width)
    gamma, beta = 1 + 0.1 * randn(g, width), randn(g, width)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ops.layer_norm(x, gamma, beta, 1e-5, y, mean, rstd)
    assert torch.equal(mean, values.float())
    assert torch.equal(y, beta.to(kind).expand(rows, width))
    # Of the squares there is left what two sums of the first mean's errors squared (50 units in the last place, for 32 terms one after another
    # and a tree) differ by in rounding; four units in the last place are the root's.
    left = 2.0 ** -22 * (50 * 2.0 ** -23 * values.double()).square()
    assert ((rstd.double() * math.sqrt(1e-5) - 1).abs() <= 2.0 ** -22 + 2.0 ** -24 + 0.5 * left / 1e-5).all()


@kinds
@pytest.mark.parametrize("width", [128, 256, 512, 1024, 2048, 4096, 8192, 100, 1000, 5001, 9000])
def test_equal_values_of_a_row_stay_equal(ops, kind, width):
    """A row has one mean and one rstd: columns of one value give one result, whichever thread works on them, and the statistics that are
    stored are the ones that were used."""
    g = gen(width)
    table = randn(g, 16).to(kind)
    pick = torch.randint(0, 16, (6, width), generator=g, device=DEV)
    x = table[pick]
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    ops.layer_norm(x, None, None, 1e-5, y, mean, rstd)
    for r in range(6):
        for v in range(16):
            got = y[r][pick[r] == v]
            assert (got == got[:1]).all(), (r, v)
    # (x - mean) * rstd + 0 in fp32: two roundings, the same here
    assert torch.equal(y, ((x.float() - mean[:, None]) * rstd[:, None]).to(kind))


# ---- orthogonalised update --------------------------------------------------------------------------------------
@kinds
@pytest.mark.parametrize("rows,cols", [(24, 40), (40, 24), (140, 200), (200, 140)])
@pytest.mark.parametrize("co,steps,scale", [((60.0, 10.0, 10.0), 1, 0.25), ((60.0, 10.0, 10.0), 2, 2.0 ** -30), ((63.0, 63.0, 63.0), 1, 1.0),
                                            ((20.0, 0.0, 0.0), 3, 2.0 ** -8), ((-63.0, 63.0, 0.0), 1, 1.0), ((1.0, -63.0, 63.0), 2, 1.0)])
def test_large_coefficients(ops, kind, rows, cols, co, steps, scale):
    """Iterates and polynomials beyond 64, from matrices of one entry, for which every product is one term: X0 is exactly 1. Each step
    rounds A, B and X once (one fp16 plane 2^-11, two 2^-22) and evaluates B in fp32. Errors of X enter the next one five times, of A twice."""
    g = torch.zeros(2, rows, cols, device=DEV)
    g[0, 3, 5] = 0.5
    g[1, 7, 2] = -4.0
    out = torch.empty(2, rows, cols, device=DEV, dtype=kind)
    ops.orthogonalise(g, out, steps=steps, coefficients=co, eps=0.0, scale=scale)
    want = ob.newton_schulz(g.double(), steps, [co], 0.0, scale)
    u = 2.0 ** -22 if kind == torch.float32 else 2.0 ** -11
    tol = sum(5.0 ** i * (4 * u + 2.0 ** -21) for i in range(steps)) + ob.U[kind]
    ob.check(out, want, tol * want.abs(), "one entry")


@kinds
@pytest.mark.parametrize("rows,cols", [(24, 40), (140, 200)])
def test_coefficients_of_each_step(ops, kind, rows, cols):
    """A step that makes the singular values large and one that brings them back: the scale follows them up and down."""
    co = [(40.0, 0.0, 0.0), (0.025, 0.0, 0.0), (1.875, -1.25, 0.375)]
    g = randn(gen(rows), 3, rows, cols)
    out = torch.empty(3, rows, cols, device=DEV, dtype=kind)
    ops.orthogonalise(g, out, steps=3, coefficients=co)
    exact = ob.newton_schulz(g.double(), 3, co, 1e-7)
    # three roundings of X on the way, two of B that matter (multiples of the identity), and the sums'
    u = 2.0 ** -20 if kind == torch.float32 else 2.0 ** -11
    off, norm = (out.double() - exact).flatten(1).norm(dim=1), exact.flatten(1).norm(dim=1)
    assert (off <= (8 * u + 2 * ob.U[kind]) * norm).all(), off / norm


@pytest.mark.parametrize("batch,rows,cols", [(16, 16, 16), (8, 24, 40), (8, 64, 256), (8, 256, 64), (8, 100, 90), (4, 128, 512), (4, 128, 128), (4, 30, 2000),
                                             (2, 300, 200), (2, 511, 700)])
def test_fp32_results_have_the_accuracy_of_fp32_products(ops, batch, rows, cols):
    """Against the same iteration with plain fp32 products: half as much again, and 2^-22 for each of the three matrices of a step that
    are held in two planes."""
    g = gen(rows * cols)
    x = randn(g, batch, rows, cols) * (torch.rand(batch, rows, cols, generator=g, device=DEV) < 0.2)
    x = x + 0.11 * randn(g, batch, rows, 4) @ randn(g, batch, 4, cols)
    out = torch.empty_like(x)
    ops.orthogonalise(x, out)
    exact = ob.newton_schulz(x.double(), 5, [(3.4445, -4.7750, 2.0315)], 1e-7)
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        plain = ob.newton_schulz(x, 5, [(3.4445, -4.7750, 2.0315)], 1e-7)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before
    norm = exact.norm()
    assert (out.double() - exact).norm() / norm <= 1.5 * (plain.double() - exact).norm() / norm + 3 * 2.0 ** -22


# ---- arguments that share memory ---------------------------------------------------------------------------------
def test_outputs_that_are_parameters_are_refused(ops):
    """Whatever is written, with no rows or tokens at all too, is none of the parameters; nothing is launched."""
    L, h = sc.operators.lib(), ops._h
    bufs = [torch.full((64, 64), 7.0, device=DEV) for _ in range(8)]
    p, q, r, s, t, u, v, w = [x.data_ptr() for x in bufs]
    for mean, rstd in ((r, None), (None, r), (s, None), (None, s)):
        assert L.scalecom_layer_norm(h, 0, 8, 8, p, 8, r, s, 1e-5, q, 8, mean, rstd) == b.ERR_ALIAS
    for rows in (0, 8):
        for dg, db in ((r, None), (None, r), (r, s)):
            assert L.scalecom_layer_norm_backward(h, 0, rows, 8, p, 8, q, 8, r, t, u, None, 8, dg, db) == b.ERR_ALIAS
    for tokens in (0, 8):
        for grads in ((r, None, None), (s, None, None), (None, t, None), (None, r, None), (None, None, t), (None, None, s)):
            assert L.scalecom_gated_ffn_backward(h, 0, 0, 0, tokens, 8, 8, p, 8, q, 8, r, s, t, u, None, 8, *grads) == b.ERR_ALIAS
    torch.cuda.synchronize()
    assert all((x == 7.0).all() for x in bufs)


# ---- CUDA graphs -------------------------------------------------------------------------------------------------
def _block(o, t, d, f, seed):
    g = gen(seed)
    x, dy = randn(g, t, d), randn(g, t, d)
    w = [randn(g, f, d) / d ** 0.5, randn(g, f, d) / d ** 0.5, randn(g, d, f) / f ** 0.5]
    y, saved, grads = torch.empty_like(x), torch.empty(2, t, f, device=DEV), [torch.empty_like(v) for v in (x, *w)]

    def call():
        o.gated_ffn(x, *w, y, saved=saved)
        o.gated_ffn_backward(dy, x, *w, saved, *grads)
    return call, [y, saved, *grads]


def test_a_graph_keeps_the_scratch_it_was_captured_with():
    """Calls that need more scratch come between a graph's replays; what is allocated meanwhile is not written over."""
    s = torch.cuda.Stream()
    with sc.Operators(stream=s) as o:
        work, outs = _block(o, 64, 128, 256, 1)
        torch.cuda.synchronize()
        work()
        s.synchronize()
        want = [v.clone() for v in outs]
        graphs, held = [], []
        for t in (64, 300, 1200):                                   # each larger than the one before
            more, _ = _block(o, t, 128, 256, t)
            torch.cuda.synchronize()
            more()
            s.synchronize()
            held.append(o.workspace())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                work()
            graphs.append(graph)
        assert held == sorted(held) and held[0] < held[2]
        fill = [torch.full((1 << 20,), 7.0, device=DEV) for _ in range(64)]
        for graph in graphs + graphs[::-1]:
            for v in outs:
                v.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(v, w) for v, w in zip(outs, want))
        assert all((v == 7.0).all() for v in fill)
        assert o.status() == 0


def test_scratch_cannot_grow_while_a_stream_is_captured():
    s = torch.cuda.Stream()
    with sc.Operators(stream=s) as o:
        work, outs = _block(o, 64, 128, 256, 1)
        n = torch.zeros(4, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            n += 1
            with pytest.raises(sc.ScaleComError) as e:
                work()
            n += 1
        assert e.value.code == b.ERR_BAD_STATE
        graph.replay()                                              # the capture went on
        torch.cuda.synchronize()
        assert (n == 2).all()
        work()                                                      # and the handle takes calls
        assert o.status() == 0 and o.workspace() > 0
