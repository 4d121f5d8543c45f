"""A two-layer network whose weights live as low-rank factors and 8-bit codes, trained on a planted teacher.

    python examples/mlp_from_svd.py [--features 1024 --hidden 4096 --tokens 2048 --rank 64 --steps 8 --type bf16]

Each weight is decomposed once by rsvd_run, W = U Vt + rest; the rest is held in 8 bits (rsvd_q8_rows).  A step runs
    forward    rsvd_q8_product of both layers; their inputs are kept in 8 bits for the backward pass (rsvd_keep8_save)
    backward   rsvd_q8_product_grad for the activations, rsvd_keep8_grad for weights and biases (added up over two half batches); the
               activation function's derivative comes from the kept numbers (rsvd_keep8_load)
    update     of the fp32 weights that the trainer holds; the factors stay, the rest is put into 8 bits again
and the trained network then answers a single token (the same rsvd_q8_product).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2110_03423_amd import Rsvd, Weight8  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


class Layer:
    """A weight (fp32, m x n) with the bias, and what the products take: factors of its largest part and the rest as codes."""

    def __init__(self, ctx, W, bias, rank):
        self.ctx, self.W, self.bias = ctx, W, bias
        S, U, Vt, _ = ctx.rsvd_run(W, rank, 16, 2, want_info=False)
        root = S.sqrt()
        self.U, self.Vt = (U * root).bfloat16().contiguous(), (root[:, None] * Vt).bfloat16().contiguous()
        self.dW, self.db = torch.empty_like(W), torch.empty_like(bias)
        self.lay_out()

    def lay_out(self):
        rest = self.W - self.U.float() @ self.Vt.float()
        codes, scale = self.ctx.rsvd_q8_rows(rest)
        self.weight = Weight8(codes, scale, self.U, self.Vt, self.bias)

    def forward(self, X, keep=True):
        kept = self.ctx.rsvd_keep8_save(X) if keep else None
        return self.ctx.rsvd_q8_product(X, self.weight), kept

    def backward(self, dY, kept, accumulate, want_dx=True):
        self.ctx.rsvd_keep8_grad(dY, kept, out=(self.dW, self.db), accumulate=accumulate)
        return self.ctx.rsvd_q8_product_grad(dY, self.weight) if want_dx else None

    def update(self, rate):
        self.W -= rate * self.dW
        self.bias -= rate * self.db
        self.lay_out()


class Mlp:
    """y = W2 relu(W1 x + b1) + b2"""

    def __init__(self, ctx, W1, b1, W2, b2, rank):
        self.ctx, self.first, self.second = ctx, Layer(ctx, W1, b1, rank), Layer(ctx, W2, b2, rank)

    def forward(self, X, keep=True):
        H, kept_x = self.first.forward(X, keep)
        H = torch.relu(H)
        Y, kept_h = self.second.forward(H, keep)
        return Y, (kept_x, kept_h)

    def backward(self, dY, kept, accumulate):
        kept_x, kept_h = kept
        dH = self.second.backward(dY, kept_h, accumulate)
        dH = torch.where(self.ctx.rsvd_keep8_load(kept_h) > 0, dH, 0)      # (a code that rounded to 0 counts as not active)
        self.first.backward(dH.contiguous(), kept_x, accumulate, want_dx=False)

    def step(self, X, target, rate, parts=2):
        """One step on the mean squared error, the batch in `parts` parts; returns the error before it."""
        total = 0.0
        for i, (x, t) in enumerate(zip(X.chunk(parts), target.chunk(parts))):
            Y, kept = self.forward(x)
            diff = Y.float() - t
            total += float((diff * diff).sum())
            self.backward(diff.to(x.dtype), kept, accumulate=i > 0)      # (of half the sum of squares: the mean's would be small for fp16)
        self.first.update(rate * 2 / target.numel())
        self.second.update(rate * 2 / target.numel())
        return total / target.numel()


def network(features, hidden, seed, device="cuda"):
    """Weights with a decaying spectrum and small biases."""
    g = torch.Generator(device=device).manual_seed(seed)

    def weight(m, n):
        k = min(m, n, 64)
        a, b = torch.randn(m, k, generator=g, device=device), torch.randn(k, n, generator=g, device=device)
        decay = 0.9 ** torch.arange(k, device=device)
        return ((a * decay) @ b / (decay.norm() * n ** 0.5) + 0.3 * torch.randn(m, n, generator=g, device=device) / n ** 0.5).contiguous()

    return (weight(hidden, features), 0.1 * torch.randn(hidden, generator=g, device=device),
            weight(features, hidden), 0.1 * torch.randn(features, generator=g, device=device))


def train(features=1024, hidden=4096, tokens=2048, rank=64, steps=8, dtype=torch.bfloat16, rate=None, seed=0):
    """Errors before each step and after the last, the trained network and its answer to the first token alone."""
    ctx = Rsvd(0)
    W1, b1, W2, b2 = network(features, hidden, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    X = torch.randn(tokens, features, generator=g, device="cuda").to(dtype)
    target = torch.relu(X.float() @ W1.t() + b1) @ W2.t() + b2
    net = Mlp(ctx, W1 + 0.02 * torch.randn(W1.shape, generator=g, device="cuda"), b1.clone(),
              W2 + 0.02 * torch.randn(W2.shape, generator=g, device="cuda"), b2.clone(), rank)
    rate = features / hidden if rate is None else rate      # (the second weight's curvature is about hidden / features)
    errors = [net.step(X, target, rate) for _ in range(steps)]
    Y, _ = net.forward(X, keep=False)
    errors.append(float(((Y.float() - target) ** 2).mean()))
    one, _ = net.forward(X[:1], keep=False)
    return errors, net, Y, one


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--features", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--rank", type=int, default=64)
    p.add_argument("--steps", type=int, default=8)
    p.add_argument("--type", choices=sorted(TYPES), default="bf16")
    a = p.parse_args()
    errors, net, Y, one = train(a.features, a.hidden, a.tokens, a.rank, a.steps, TYPES[a.type])
    for i, e in enumerate(errors):
        print(f"step {i}: mean squared error {e:.6f}")
    full = 4 * (net.first.W.numel() + net.second.W.numel())
    held = sum(w.codes.numel() + 4 * w.m + 2 * w.r * (w.m + w.n) for w in (net.first.weight, net.second.weight))
    print(f"weights: {full / 1e6:.1f} MB in fp32, {held / 1e6:.1f} MB as factors and codes")
    print(f"one token alone against the same in the batch: largest difference {float((one - Y[:1]).float().abs().max()):.3g}")


if __name__ == "__main__":
    main()
