"""Trains a small residual MLP that predicts the next token of a synthetic language, with every gradient from this package:

    python examples/train_residual_mlp.py [--steps 60] [--width 256] [--layers 2] [--classes 4096] [--tokens 2048]

A layer is   z = h W1,  f = gelu(z) W2,  r <- r + scale gate norm_post(f),  h = norm_pre(r).
Kept for the backward pass are 8-bit checkpoints of h, z, r and f (shampoo_checkpoint_pack, shampoo_residual_norm_forward).  The
head's loss and its gradients come from shampoo_linear_cross_entropy, the layers' from shampoo_residual_norm_backward,
shampoo_checkpoint_weight_grad and shampoo_checkpoint_activation_grad, and Shampoo.step takes them all: bf16 gradients for
the matrices, in one optimizer, and float32 ones for gates and norm weights in another."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_06497_amd import binding as B  # noqa: E402


class ResidualMLP:
    SCALE = 0.5

    def __init__(self, classes, width, layers, seed=0, device=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        normal = lambda *shape: torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[0])
        self.layers = layers
        self.embed = normal(classes, width).mul_(math.sqrt(classes)).bfloat16()                    # not trained
        # matrices [in, out], and the head [classes, width]; per layer two vectors after the block and one before the next
        self.matrices = [m for _ in range(layers) for m in (normal(width, 4 * width), normal(4 * width, width))] + [normal(classes, width) * 0.05]
        one = lambda: torch.ones(width, device="cuda")
        self.vectors = [v for _ in range(layers) for v in (one(), one(), one())]                   # gate, w_post, w_pre
        shapes = lambda tensors: [tuple(t.shape) for t in tensors]
        self.opt = B.Shampoo(shapes(self.matrices), 1024, 0.99, 1e-8, 0.25, 10, 0, 1e-8, 0.9, grad_dtype=B.GRAD_BF16, device=device)
        self.opt_vectors = B.Shampoo(shapes(self.vectors), 1024, 0.99, 1e-8, 0.25, 10, 0, 1e-8, 0.9, device=device)

    def loss_and_gradients(self, tokens, targets):
        """Mean loss (a tensor), and the gradients of matrices and vectors"""
        n = tokens.shape[0]
        w = [m.bfloat16() for m in self.matrices]
        r = self.embed[tokens]
        h, kept = r, []
        for i in range(self.layers):
            gate, w_post, w_pre = self.vectors[3 * i:3 * i + 3]
            z = h @ w[2 * i]
            f = torch.nn.functional.gelu(z) @ w[2 * i + 1]
            h8, z8 = B.shampoo_checkpoint_pack(h), B.shampoo_checkpoint_pack(z)
            r, h, r8, f8 = B.shampoo_residual_norm_forward(r, f, gate=gate, w_post=w_post, w_pre=w_pre, scale=self.SCALE, checkpoint=True)
            kept.append((h8, z8, r8, f8))
        loss, dh, dw, _ = B.shampoo_linear_cross_entropy(h, w[-1], targets, scale=1.0 / n)
        matrices, vectors, dr = [dw], [], None
        for i in reversed(range(self.layers)):
            gate, w_post, w_pre = self.vectors[3 * i:3 * i + 3]
            h8, z8, r8, f8 = kept.pop()
            g = B.shampoo_residual_norm_backward(r8, f8, dr, dh, gate=gate, w_post=w_post, w_pre=w_pre, scale=self.SCALE)
            dr, df = g["dr"], g["df"]
            dw2 = B.shampoo_checkpoint_weight_grad(z8, df, B.ACT_GELU)
            dz = B.shampoo_checkpoint_activation_grad(z8, df @ w[2 * i + 1].t(), B.ACT_GELU)
            dw1 = B.shampoo_checkpoint_weight_grad(h8, dz)
            dh = dz @ w[2 * i].t()
            matrices = [dw1, dw2] + matrices
            vectors = [g["dgate"], g["dw_post"], g["dw_pre"]] + vectors
        return loss.mean(), matrices, vectors

    def step(self, tokens, targets, lr, t):
        loss, matrices, vectors = self.loss_and_gradients(tokens, targets)
        self.opt.step(self.matrices, matrices, lr, t)
        self.opt_vectors.step(self.vectors, vectors, lr, t)
        return loss


def batch(classes, tokens, seed):
    """A language in which every token has one likely successor"""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randint(0, classes, (tokens,), generator=g, device="cuda")
    noise = torch.randint(0, classes, (tokens,), generator=g, device="cuda")
    return x, torch.where(torch.rand((tokens,), generator=g, device="cuda") < 0.9, (x * 7 + 3) % classes, noise)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 60), ("width", 256), ("layers", 2), ("classes", 4096), ("tokens", 2048)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    model = ResidualMLP(a.classes, a.width, a.layers)
    for t in range(a.steps):
        loss = model.step(*batch(a.classes, a.tokens, t), 0.02, t)
        if t % 10 == 0 or t == a.steps - 1:
            print(f"step {t:4d}  loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
