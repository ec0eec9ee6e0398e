"""The example that runs layer norm, the gated block, the CLT-k step and the orthogonalised update together."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.mark.parametrize("kind", [torch.float32, torch.float16, torch.bfloat16], ids=["f32", "f16", "bf16"])
def test_learners_train(kind):
    import learners
    a = learners.train(kind, steps=60)
    assert all(v == v for v in a)
    assert sum(a[-5:]) < 0.5 * sum(a[:5])                 # the loss is at least halved
    b = learners.train(kind, steps=3)
    assert b == a[:3]                                     # the same run gives the same losses


def test_block_gradient_in_a_flat_vector_matches_autograd():
    """The whole block's gradient, layer norm included, against automatic differentiation in 64 bits."""
    import learners
    import paper_2104_11125_b200 as sc
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(4)
    with sc.Operators() as ops:
        block = learners.Block(40, 72, torch.float32, ops)
        flat = torch.randn(block.size, generator=gen, device="cuda:0") * 0.2
        grad = torch.empty(block.size, device="cuda:0")
        x = torch.randn(33, 40, generator=gen, device="cuda:0")
        target = torch.randn(33, 40, generator=gen, device="cuda:0")
        block.gradient(block.slices(flat), x, target, block.slices(grad))
        leaf = flat.double().requires_grad_()
        w = block.slices(leaf)
        z = torch.nn.functional.layer_norm(x.double(), (40,), w["gamma"], w["beta"], 1e-5)
        y = x.double() + (torch.nn.functional.silu(z @ w["w_gate"].t()) * (z @ w["w_up"].t())) @ w["w_down"].t()
        ((y - target.double()).square().sum() / 40).backward()
        # five chained fp32 stages of at most 72 terms: some 2^-18 of the gradient's size
        assert (grad.double() - leaf.grad).norm() < 2.0 ** -18 * leaf.grad.norm()
        assert ops.status() == 0
