"""Trains a small feed-forward block with the library's layers and serves a mixture of experts with them.

Training: two linear layers with a gelu between them, their gradients, and AdamW on float weights with moments in 8 bits and a
bfloat16 copy that the products read.  Serving: one token at a time through a mixture-of-experts layer.

    python examples/feed_forward.py [--steps 200]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2506_11277_amd import layers


class FeedForward:
    """y = x + gelu(x w1^T + b1) w2^T + b2, trained on a target."""

    def __init__(self, width, hidden, bits=8):
        def normal(*shape, std):
            return torch.randn(*shape, device="cuda").mul_(std)

        self.masters = [normal(hidden, width, std=width ** -0.5), torch.zeros(hidden, device="cuda"),
                        normal(width, hidden, std=hidden ** -0.5), torch.zeros(width, device="cuda")]
        self.weights = [m.to(torch.bfloat16) for m in self.masters]
        self.plan = layers.AdamW(self.masters, *layers.adamw_state(self.masters, bits), copies=self.weights)
        self.steps = 0

    def forward(self, x):
        w1, b1, w2, b2 = self.weights
        self.x, self.pre = x, torch.empty((x.shape[0], w1.shape[0]), dtype=x.dtype, device=x.device)
        self.h = layers.linear(x, w1, b1, activation=layers.ACT_GELU, pre=self.pre)
        return layers.linear(self.h, w2, b2, residual=x)

    def step(self, dy, lr):
        dh, dw2, db2 = layers.linear_grad(dy, self.h, self.weights[2])
        _, dw1, db1 = layers.linear_grad(dh, self.x, self.weights[0], self.pre, layers.ACT_GELU, want=("dw",))
        self.steps += 1
        self.plan.step([dw1, db1, dw2, db2], self.steps, lr=lr, weight_decay=0.0, seed=self.steps)


def train(steps, tokens=512, width=256, hidden=1024, bits=8):
    """Losses of a block that learns another block's map."""
    torch.manual_seed(0)
    teacher, student = FeedForward(width, hidden), FeedForward(width, hidden, bits)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
        error = student.forward(x).float() - teacher.forward(x).float()
        losses.append(error.square().mean())
        student.step((error * (2.0 / width)).to(torch.bfloat16), lr=1e-3)
    return torch.stack(losses).tolist()


def serve(tokens=8, width=512, hidden=256, experts=16, top_k=2):
    """Token after token through a residual mixture-of-experts layer; the results' norms and the experts taken."""
    torch.manual_seed(1)
    bf16 = torch.bfloat16
    router = torch.randn(experts, width, device="cuda").mul_(width ** -0.5).to(bf16)
    w_in = torch.randn(experts, 2 * hidden, width, device="cuda").mul_(width ** -0.5).to(bf16)
    w_out = torch.randn(experts, width, hidden, device="cuda").mul_(hidden ** -0.5).to(bf16)
    x = torch.randn(1, width, device="cuda").to(bf16)
    norms, taken = [], []
    for _ in range(tokens):
        scaled = x * x.float().square().mean(-1, keepdim=True).rsqrt().to(bf16)
        y, chosen, _ = layers.moe(scaled, router, w_in, w_out, top_k)
        x = x + y
        norms.append(x.float().norm())
        taken.append(chosen)
    return torch.stack(norms).tolist(), torch.cat(taken).tolist()


def main():
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=200)
    steps = parser.parse_args().steps
    losses = train(steps)
    print(f"training: loss {losses[0]:.4f} at the first step, {losses[-1]:.4f} at step {steps}")
    norms, taken = serve()
    print(f"serving: {len(taken)} tokens, experts {taken}, norms {[round(n, 2) for n in norms]}")


if __name__ == "__main__":
    main()
