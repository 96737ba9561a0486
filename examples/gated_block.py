#!/usr/bin/env python3
"""A pre-norm gated feed-forward block, trained and then served.

Training: y = silu(n Wg^T) * (n Wu^T) Wd^T + b + x with n = norm(x) learns the function of a block of the same shape.
Between forward and backward pass the block keeps n and both projections as 8-bit floats with one
power-of-two scale a group of 32, 1.03 bytes a value; its optimiser keeps both moments so as well. The weights are
float32 for the optimiser, which writes the bfloat16 copies that the products read.

Serving: the trained weights go to 4-bit floats with one scale a group, and tokens run through the
block one at a time: one launch for the norm, one for both projections, the activation and the product, one for the
last projection.

    python examples/gated_block.py [--tokens 512] [--width 512] [--hidden 1408] [--steps 80]
"""
import argparse
import os
import sys

import torch
from torch.autograd.function import once_differentiable

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2007_06563_amd import hobflops as hf  # noqa: E402

E4M3, E2M1 = (4, 3), (2, 1)


class Gated(torch.autograd.Function):
    """act(x w_gate^T) * (x w_up^T), whose backward pass starts from 8-bit checkpoints. It has no second
    derivative: asking for one is an error."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up):
        h, saved = hf.gated_forward(x, w_gate, w_up, hf.GATE_SILU, ckpt=E4M3)
        ctx.fmt = saved.fmt
        ctx.save_for_backward(*saved.x, *saved.gate, *saved.up, w_gate, w_up)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        t = ctx.saved_tensors
        saved = hf.GatedSaved(t[0:2], t[2:4], t[4:6], ctx.fmt)
        return hf.gated_backward(dh.contiguous(), saved, t[6], t[7], hf.GATE_SILU)


class Norm(torch.autograd.Function):
    """Layer norm."""

    @staticmethod
    def forward(ctx, x, weight, bias):
        y, saved = hf.layer_norm(x, weight, bias, save=True)
        ctx.save_for_backward(x, weight, *saved)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, *saved = ctx.saved_tensors
        return hf.layer_norm_backward(dy.contiguous(), x, hf.NormSaved(*saved), weight)


class Projection(torch.autograd.Function):
    """x w^T + bias + residual."""

    @staticmethod
    def forward(ctx, x, w, bias, residual):
        ctx.save_for_backward(x, w)
        return hf.linear(x, w, bias, residual=residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        dy = dy.contiguous()
        return (*hf.linear_backward(dy, *ctx.saved_tensors), dy)


class Block:
    """float32 weights, the bfloat16 copies that the products read, 8-bit moments."""

    def __init__(self, width, hidden, generator):
        dev = generator.device

        def weight(rows, cols):
            return torch.randn(rows, cols, generator=generator, device=dev) * cols ** -0.5

        self.weights = [torch.ones(width, device=dev), torch.zeros(width, device=dev), weight(hidden, width),
                        weight(hidden, width), weight(width, hidden), torch.zeros(width, device=dev)]
        self.copies = [w.bfloat16().requires_grad_() for w in self.weights]
        self.state = hf.adamw_state(self.weights, E4M3)
        self.steps = 0

    def __call__(self, x):
        scale, shift, gate, up, down, bias = self.copies
        h = Gated.apply(Norm.apply(x, scale, shift), gate, up)
        return Projection.apply(h, down, bias, x)

    def step(self, lr):
        """One AdamW step from the copies' gradients."""
        self.steps += 1
        hf.adamw(self.weights, [c.grad for c in self.copies], self.state, self.steps, lr=lr, weight_decay=0.0,
                 copies=self.copies, seed=1)
        for c in self.copies:
            c.grad = None


class Served:
    """The block with 4-bit weights, for a few tokens at a time."""

    def __init__(self, block, group=32):
        self.group = group
        self.scale, self.shift, *weights, self.bias = (c.detach() for c in block.copies)
        self.gate, self.up, self.down = (hf.block_pack(w, E2M1, group=group, scale=hf.SCALE_BF16) for w in weights)

    def __call__(self, x):
        n = hf.layer_norm(x, self.scale, self.shift)
        h = hf.w4_gated(n, *self.gate, *self.up, hf.GATE_SILU, group=self.group)
        return hf.w4_linear(h, *self.down, group=self.group) + self.bias + x

    def bytes(self):
        return sum(t.numel() * t.element_size() for w in (self.gate, self.up, self.down) for t in w)


def run(tokens=512, width=512, hidden=1408, steps=80, served=8, say=print):
    """Trains and serves; returns (first loss, last loss, relative error of the served block)."""
    g = torch.Generator(device="cuda").manual_seed(0)
    teacher, block = Block(width, hidden, g), Block(width, hidden, g)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
        with torch.no_grad():
            want = teacher(x)
        loss = (block(x).float() - want.float()).square().mean()
        loss.backward()
        block.step(lr=2e-3)
        losses.append(loss.item())
        if step % 20 == 0 or step == steps - 1:
            say(f"step {step}: loss {losses[-1]:.4f}")
    kept = tokens * (width + 2 * hidden)
    values = sum(w.numel() for w in block.weights)
    say(f"kept for the optimiser: {values * 2 * 33 / 32 / 2 ** 20:.2f} MiB ({values * 8 / 2 ** 20:.2f} in float32)")
    say(f"kept for the backward pass: {kept * 33 / 32 / 2 ** 20:.2f} MiB "
        f"({kept * 2 / 2 ** 20:.2f} in bfloat16)")

    quick = Served(block)
    x = torch.randn(served, width, generator=g, device="cuda").bfloat16()
    with torch.no_grad():
        want = block(x).float()
    got = torch.cat([quick(x[i:i + 1]) for i in range(served)]).float()
    error = ((got - want).norm() / want.norm()).item()
    weights = 3 * width * hidden
    say(f"served from {quick.bytes() / 2 ** 20:.2f} MiB of weights ({weights * 2 / 2 ** 20:.2f} in "
        f"bfloat16): {error:.3f} off, relative")
    return losses[0], losses[-1], error


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1408)
    ap.add_argument("--steps", type=int, default=80)
    a = ap.parse_args()
    run(a.tokens, a.width, a.hidden, a.steps)
