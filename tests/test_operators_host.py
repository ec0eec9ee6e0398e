"""Host side of the learner-side operators: exported symbols, constants, and refusals that need no GPU."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2104_11125_b200 import build, operators
    build.build()
    return operators.lib()


def _header():
    return open(os.path.join(ROOT, "include", "scalecom_operators.h")).read()


def test_library_exports_every_declared_operator(lib):
    from paper_2104_11125_b200 import operators
    text = re.sub(r"/\*.*?\*/", "", _header(), flags=re.S)
    declared = set(re.findall(r"\b(scalecom_[a-z_]+)\s*\(", text))
    assert declared == set(operators.EXPORTS)
    for name in declared:
        assert getattr(lib, name) is not None


def test_constants_equal_the_header_defines():
    from paper_2104_11125_b200 import operators
    found = re.findall(r"#define\s+SCALECOM_((?:F32|F16|BF16|ACT_[A-Z_]+))\s+(\d+)", _header())
    assert len(found) == 7
    for name, value in found:
        assert getattr(operators, name) == int(value)
    assert "SCALECOM_OPS_MAX_DIM (1 << 26)" in _header() and operators.OPS_MAX_DIM == 1 << 26


def test_null_handles_are_reported(lib):
    from paper_2104_11125_b200 import binding as b
    n = ctypes.c_int64()
    assert lib.scalecom_ops_create(None) == b.ERR_NULL_PTR
    assert lib.scalecom_ops_set_stream(None, None) == b.ERR_NULL_PTR
    assert lib.scalecom_ops_reserve(None, 1) == b.ERR_NULL_PTR
    assert lib.scalecom_ops_workspace(None, ctypes.byref(n)) == b.ERR_NULL_PTR
    assert lib.scalecom_ops_status(None) == b.ERR_NULL_PTR
    assert lib.scalecom_ops_reset(None) == b.ERR_NULL_PTR
    assert lib.scalecom_layer_norm(None, 0, 1, 1, None, 1, None, None, 0.0, None, 1, None, None) == b.ERR_NULL_PTR
    assert lib.scalecom_layer_norm_backward(None, 0, 1, 1, None, 1, None, 1, None, None, None, None, 1, None, None) == b.ERR_NULL_PTR
    assert lib.scalecom_gated_ffn(None, 0, 0, 1, 1, 1, None, 1, None, None, None, None, 1, None) == b.ERR_NULL_PTR
    assert lib.scalecom_gated_ffn_backward(None, 0, 0, 0, 1, 1, 1, None, 1, None, 1, None, None, None, None, None, 1,
                                           None, None, None) == b.ERR_NULL_PTR
    assert lib.scalecom_orthogonalise(None, 1, 1, 1, 0, None, 1, 1, 0, None, 1, 1, 5, None, 1, 0.0, 1.0) == b.ERR_NULL_PTR
    lib.scalecom_ops_destroy(None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a GPU")
def test_creation_without_a_device_is_an_error(lib):
    import paper_2104_11125_b200 as sc
    with pytest.raises(sc.ScaleComError) as e:
        sc.Operators()
    assert e.value.code == sc.binding.ERR_CUDA


def test_the_binding_refuses_host_tensors_before_it_calls(lib):
    from paper_2104_11125_b200.operators import Operators
    ops = Operators.__new__(Operators)               # no handle: every call has to stop at its arguments
    x = torch.zeros(2, 4)
    with pytest.raises(TypeError):
        ops.layer_norm(x, None, None, 1e-5, x)
    with pytest.raises(TypeError):
        ops.gated_ffn(x, x, x, x, x)
    with pytest.raises(TypeError):
        ops.orthogonalise(x, x)
    with pytest.raises(ValueError):
        ops.orthogonalise(x, torch.zeros(4, 2))


def test_the_64_bit_forms_agree_with_automatic_differentiation():
    """The bounds' own reference: gradients against differentiation of the forward formula, and against differences."""
    from tests import operator_bounds as ob
    torch.manual_seed(3)
    t, d, f = 5, 7, 6
    for name in ("silu", "gelu", "gelu_tanh", "relu"):
        leaf = [torch.randn(*s, dtype=torch.float64, requires_grad=True) for s in ((t, d), (f, d), (f, d), (d, f))]
        dy = torch.randn(t, d, dtype=torch.float64)
        with torch.no_grad():
            out = ob.ffn(*leaf, name, torch.float32, dy, torch.float32)
        x, wg, wu, wd = leaf
        y = (ob.act(name, x @ wg.t())[0] * (x @ wu.t())) @ wd.t()
        y.backward(dy)
        for key, v in zip(("dx", "dw_gate", "dw_up", "dw_down"), leaf):
            assert torch.allclose(out[key][0], v.grad, rtol=1e-10, atol=1e-12), (name, key)
        with torch.no_grad():
            v, h = torch.randn(t, d, dtype=torch.float64), 1e-6
            up = ob.ffn(x + h * v, wg, wu, wd, name, torch.float32)["y"][0]
            down = ob.ffn(x - h * v, wg, wu, wd, name, torch.float32)["y"][0]
            assert abs(((up - down) / (2 * h) * dy).sum() - (out["dx"][0] * v).sum()) < 1e-6
    x = torch.randn(4, 9, dtype=torch.float64, requires_grad=True)
    gamma = torch.randn(9, dtype=torch.float64, requires_grad=True)
    beta = torch.randn(9, dtype=torch.float64, requires_grad=True)
    y = torch.nn.functional.layer_norm(x, (9,), gamma, beta, 1e-5)
    dy = torch.randn_like(y)
    y.backward(dy)
    with torch.no_grad():
        fwd = ob.layer_norm(x, gamma, beta, 1e-5, torch.float32)
        assert torch.allclose(fwd["y"][0], y, atol=1e-12)
        out = ob.layer_norm_backward(dy, x, gamma, fwd["mean"][0], fwd["rstd"][0], torch.float32)
    for key, v in (("dx", x), ("dgamma", gamma), ("dbeta", beta)):
        assert torch.allclose(out[key][0], v.grad, atol=1e-11), key


def test_the_64_bit_newton_schulz_acts_on_singular_values_alone():
    from tests import operator_bounds as ob
    torch.manual_seed(5)
    co = [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5)]
    for shape in ((2, 5, 9), (2, 9, 5)):
        g = torch.randn(*shape, dtype=torch.float64)
        u, s, v = torch.linalg.svd(g, full_matrices=False)
        s = s / (s.square().sum(1, keepdim=True).sqrt() + 1e-7)
        for i in range(4):
            a, b, c = co[i % 2]
            s = a * s + b * s ** 3 + c * s ** 5
        want = u @ torch.diag_embed(s) @ v
        assert torch.allclose(ob.newton_schulz(g, 4, co, 1e-7), want, atol=1e-10)
