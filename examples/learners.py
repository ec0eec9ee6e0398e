"""Learners with a transformer's feed-forward block, trained with the CLT-k step and the orthogonalised update.

Each of n learners runs the residual block  y = x + W_down (act(W_gate z) * (W_up z)),  z = layer_norm(x),  on its own batch; the
backward pass writes the weight gradients straight into its flat fp32 gradient vector.  scalecom_step() picks the
leader's top-k coordinates and averages the learners' values there into the momentum (a "weights" vector with a step size
of -1); the momentum's matrices are orthogonalised and applied.  Prints the loss now and then.

    python examples/learners.py [--type bf16|f16|f32] [--steps 100]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2104_11125_b200 as sc  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Block:
    """The block's parameters as slices of one flat fp32 vector, and its two passes for one learner."""

    def __init__(self, width: int, hidden: int, kind: torch.dtype, ops: "sc.Operators"):
        self.ops, self.kind = ops, kind
        self.shapes = {"w_gate": (hidden, width), "w_up": (hidden, width), "w_down": (width, hidden), "gamma": (width,), "beta": (width,)}
        self.size = sum(torch.Size(s).numel() for s in self.shapes.values())

    def slices(self, flat: torch.Tensor) -> dict:
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def gradient(self, weights: dict, x: torch.Tensor, target: torch.Tensor, grad: dict) -> torch.Tensor:
        """Mean squared error of the block's output, and its gradient in the slices of `grad`."""
        ops, kind, (tokens, width) = self.ops, self.kind, x.shape
        dev, hidden = x.device, weights["w_gate"].shape[0]
        low = {k: weights[k].to(kind) for k in ("w_gate", "w_up", "w_down")}
        z, y = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(tokens, device=dev), torch.empty(tokens, device=dev)
        saved = torch.empty(2, tokens, hidden, device=dev, dtype=kind)
        ops.layer_norm(x, weights["gamma"], weights["beta"], 1e-5, z, mean, rstd)
        ops.gated_ffn(z, low["w_gate"], low["w_up"], low["w_down"], y, saved=saved)
        off = (x.float() + y.float()) - target
        # the gradient of the squared errors' sum over width: of the errors' own size, far from fp16's subnormals
        dy = (off * (2.0 / width)).to(kind)
        dz, dx = torch.empty_like(x), torch.empty_like(x)
        ops.gated_ffn_backward(dy, z, low["w_gate"], low["w_up"], low["w_down"], saved, dz, grad["w_gate"], grad["w_up"], grad["w_down"])
        ops.layer_norm_backward(dz, x, weights["gamma"], mean, rstd, dx, grad["gamma"], grad["beta"])
        return off.square().mean()


def train(kind: torch.dtype = torch.bfloat16, steps: int = 100, learners: int = 4, tokens: int = 512, width: int = 128, hidden: int = 256,
          lr: float = 0.02, momentum: float = 0.9, ratio: int = 20, seed: int = 1, device: str = "cuda:0", log=None) -> list:
    """Losses (mean over the learners) of every step."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    ops = sc.Operators()
    block = Block(width, hidden, kind, ops)
    weights, move = torch.empty(block.size, device=device), torch.zeros(block.size, device=device)
    w, m = block.slices(weights), block.slices(move)
    for name, v in w.items():
        v.copy_(torch.ones_like(v) if name == "gamma" else torch.zeros_like(v) if name == "beta"
                else torch.randn(v.shape, generator=gen, device=device) / v.shape[1] ** 0.5)
    goal = torch.randn(width, width, generator=gen, device=device) / width ** 0.5
    grads = [torch.empty(block.size, device=device) for _ in range(learners)]
    memory = [torch.zeros(block.size, device=device) for _ in range(learners)]
    k = block.size // ratio
    idx, val = torch.empty(k, device=device, dtype=torch.int32), torch.empty(k, device=device)
    losses = []
    with sc.Context(block.size, learners, k, 0.5, -1.0) as ctx:
        for t in range(steps):
            total = 0.0
            for i in range(learners):
                x = torch.randn(tokens, width, generator=gen, device=device).to(kind)
                total = total + block.gradient(w, x, x.float() + torch.tanh(x.float() @ goal), block.slices(grads[i]))
            move.mul_(momentum)
            ctx.step(grads, memory, move, t, idx, val)                  # move += the averaged values at the leader's indices
            for name, v in w.items():
                if v.dim() == 2:
                    step = torch.empty(v.shape, device=device, dtype=torch.bfloat16)
                    ops.orthogonalise(m[name], step, scale=max(1.0, v.shape[0] / v.shape[1]) ** 0.5)
                    v.add_(step, alpha=-lr)
                else:
                    v.add_(m[name].sign(), alpha=-0.1 * lr)
            losses.append(total / learners)
            if log and (t % 10 == 0 or t + 1 == steps):
                log("step %4d  loss %.4f" % (t, losses[-1].item()))
        if ctx.status() != 0 or ops.status() != 0:
            raise RuntimeError("a kernel reported an error")
    return [v.item() for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--type", choices=sorted(TYPES), default="bf16")
    ap.add_argument("--steps", type=int, default=100)
    a = ap.parse_args()
    train(TYPES[a.type], a.steps, log=print)
