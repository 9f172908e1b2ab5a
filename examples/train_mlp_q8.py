"""Trains a small residual MLP whose linear layers run in 8 bits, its weights with Periodic Row-wise Muon
and its norm weights with AdamW, on targets from a fixed random network of the same kind.

    python examples/train_mlp_q8.py --steps 60 --format int8      # or e4m3, or bf16 for comparison
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2608_20818_b200.binding import PeriodicRowwiseMuon, prm_adamw_step
from paper_2608_20818_b200.q8 import Weight8, linear, norm_linear

EPS = 1e-6


class Mlp:
    """Blocks of h + gelu(norm(h) @ up) @ down."""

    def __init__(self, dim, blocks, format, generator):
        def matrix(rows, cols):
            w = torch.randn(rows, cols, generator=generator, device="cuda") * rows ** -0.5
            return w.to(torch.bfloat16).requires_grad_()

        self.weights = [w for _ in range(blocks) for w in (matrix(dim, 4 * dim), matrix(4 * dim, dim))]
        self.norms = [torch.ones(dim, device="cuda", requires_grad=True) for _ in range(blocks)]
        self.eight = None if format == "bf16" else [Weight8(w, format) for w in self.weights]

    def refresh(self):
        for w in self.eight or ():
            w.refresh()

    def __call__(self, x):
        stream, update = x, None
        for i, norm in enumerate(self.norms):
            if self.eight:
                y, stream = norm_linear(stream, update, norm, self.eight[2 * i], EPS)
                update = linear(torch.nn.functional.gelu(y), self.eight[2 * i + 1])
            else:
                stream = stream if update is None else stream + update
                v = stream.float()
                n = (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * norm).to(stream.dtype)
                update = torch.nn.functional.gelu(n @ self.weights[2 * i]) @ self.weights[2 * i + 1]
        return stream + update


def train(steps=60, dim=512, blocks=2, tokens=2048, format="int8", lr=0.02, seed=0, log=print):
    """Returns the losses, step by step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    model, teacher = Mlp(dim, blocks, format, g), Mlp(dim, blocks, "bf16", g)
    optimizer = PeriodicRowwiseMuon([tuple(w.shape) for w in model.weights], K=5, beta=0.95, nesterov=True, lr=lr, wd=0.0)
    momentum = [torch.zeros(w.shape, device="cuda") for w in model.weights]
    first = [torch.zeros_like(n) for n in model.norms]
    second = [torch.zeros_like(n) for n in model.norms]
    losses = []
    for t in range(steps):
        x = torch.randn(tokens, dim, generator=g, device="cuda").to(torch.bfloat16)
        with torch.no_grad():
            target = teacher(x).float()
        loss = (model(x).float() - target).square().mean()
        loss.backward()
        with torch.no_grad():
            optimizer.step([w.detach() for w in model.weights], [w.grad for w in model.weights], momentum, t)
            prm_adamw_step([n.detach() for n in model.norms], [n.grad for n in model.norms], first, second, t + 1, lr=1e-3)
        for p in model.weights + model.norms:
            p.grad = None
        model.refresh()
        losses.append(loss.item())
        if log and (t % 10 == 0 or t + 1 == steps):
            log(f"step {t:3d}  loss {losses[-1]:.4f}")
    optimizer.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--format", choices=("int8", "e4m3", "bf16"), default="int8")
    a = ap.parse_args()
    train(a.steps, a.dim, a.blocks, a.tokens, a.format)
