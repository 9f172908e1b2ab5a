"""Trains a small next-token model on a synthetic chain of tokens: layer norm with dropout at the residual's addition,
linear layers in 8 bits, and the loss over the vocabulary without its logits.  The layers' weights take Periodic Row-wise
Muon, embedding, head and norms AdamW.

    python examples/train_tokens_q8.py --steps 60 --format int8       # or e4m3, or bf16 for comparison
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2608_20818_b200.binding import PRM_OK, PeriodicRowwiseMuon, prm_adamw_step, prm_q8_status
from paper_2608_20818_b200.layers import Draws, head_loss, layer_norm
from paper_2608_20818_b200.q8 import Weight8, linear


class Model:
    """Embedding, blocks of stream + dropout(gelu(norm(stream) @ up) @ down), a last norm, head."""

    def __init__(self, vocab, dim, blocks, format, p, generator):
        def matrix(rows, cols, std):
            w = torch.randn(rows, cols, generator=generator, device="cuda") * std
            return w.to(torch.bfloat16).requires_grad_()

        self.embedding = matrix(vocab, dim, 1.0)
        self.weights = [w for _ in range(blocks) for w in (matrix(dim, 4 * dim, dim ** -0.5), matrix(4 * dim, dim, (4 * dim) ** -0.5))]
        self.norms = [torch.full((dim,), v, device="cuda").requires_grad_() for _ in range(blocks + 1) for v in (1.0, 0.0)]
        self.head = matrix(dim, vocab, 0.5 * dim ** -0.5)
        self.p = p
        self.eight = None if format == "bf16" else [Weight8(w, format) for w in self.weights]

    def product(self, x, i):
        return linear(x, self.eight[i]) if self.eight else x @ self.weights[i]

    def refresh(self):
        for w in self.eight or ():
            w.refresh()

    def __call__(self, tokens, labels, draws):
        """The mean loss over the tokens with a label."""
        stream, update = self.embedding[tokens], None
        for i in range(len(self.norms) // 2):
            weight, bias = self.norms[2 * i:2 * i + 2]
            if update is None:
                y, stream = layer_norm(stream, weight, bias)
            else:
                y, stream = layer_norm(update, weight, bias, residual=stream, p=self.p, draws=draws)
            if 2 * i < len(self.weights):
                update = self.product(torch.nn.functional.gelu(self.product(y, 2 * i)), 2 * i + 1)
        return head_loss(y, self.head, labels).sum() / (labels >= 0).sum()


def train(steps=60, vocab=1000, dim=256, blocks=2, tokens=2048, format="int8", p=0.1, lr=0.02, seed=0, log=print):
    """Returns the losses, step by step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    model, draws = Model(vocab, dim, blocks, format, p, g), Draws(seed)
    follows = torch.randint(0, vocab, (vocab, 4), generator=g, device="cuda")      # each token has four successors
    optimizer = PeriodicRowwiseMuon([tuple(w.shape) for w in model.weights], K=5, beta=0.95, nesterov=True, lr=lr, wd=0.0)
    momentum = [torch.zeros(w.shape, device="cuda") for w in model.weights]
    others = [[model.embedding, model.head], model.norms]                         # bf16, fp32
    moments = [[[torch.zeros(t.shape, device="cuda") for t in group] for _ in range(2)] for group in others]
    losses = []
    for t in range(steps):
        x = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
        labels = follows[x, torch.randint(0, 4, (tokens,), generator=g, device="cuda")]
        labels[::16] = -100                                                        # padding
        loss = model(x, labels, draws)
        loss.backward()
        with torch.no_grad():
            optimizer.step([w.detach() for w in model.weights], [w.grad for w in model.weights], momentum, t)
            for group, (first, second) in zip(others, moments):
                prm_adamw_step([v.detach() for v in group], [v.grad for v in group], first, second, t + 1, lr=1e-2)
        for v in model.weights + others[0] + others[1]:
            v.grad = None
        model.refresh()
        draws.advance()
        losses.append(loss.item())
        if log and (t % 10 == 0 or t + 1 == steps):
            log(f"step {t:3d}  loss {losses[-1]:.4f}")
    optimizer.close()
    if prm_q8_status() != PRM_OK:
        raise RuntimeError("a wait inside a product ran out: the steps since then have wrong gradients")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--format", choices=("int8", "e4m3", "bf16"), default="int8")
    ap.add_argument("--dropout", type=float, default=0.1)
    a = ap.parse_args()
    train(a.steps, a.vocab, a.dim, a.blocks, a.tokens, a.format, a.dropout)
