"""Trains one block on a fixed batch: norm, routing, experts and the optimizer step, called as a training program calls them.

    python examples/block_step.py [--tokens 2048] [--steps 20]

The target is what another block of the same shape makes of the batch; the loss is the mean square of the difference."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_11543_amd.block import DeviceBlock  # noqa: E402


def train(tokens=2048, d_model=512, n_experts=32, d_ff=256, top_k=4, groups=4, kept_groups=2, trainable=8, steps=20, dtype="bf16", report=print):
    """The losses of `steps` steps, and the largest load of an expert relative to the mean at the first and the last."""
    shape = dict(T=tokens, d_model=d_model, n_experts=n_experts, d_ff=d_ff, top_k=top_k, groups=groups, kept_groups=kept_groups, dtype=dtype)
    mask = (np.arange(n_experts) % (n_experts // trainable) == 0).astype(np.uint8)
    block, teacher = DeviceBlock(mask=mask, seed=1, **shape), DeviceBlock(mask=np.zeros(n_experts), seed=2, **shape)
    g = torch.Generator(device="cuda").manual_seed(3)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x, add = (torch.randn(tokens, d_model, device="cuda", generator=g).to(t) for _ in range(2))
    target = teacher.forward(x, add).float()
    losses, loads = [], []
    for i in range(steps):
        diff = block.forward(x, add).float() - target
        block.backward((2 / diff.numel() * 1024 * diff).to(t))          # (a loss scale: what the optimizer makes of the gradient does not depend on it)
        block.step()
        losses.append(float(diff.square().mean()))
        loads.append(float(block.chosen.max()) / (tokens * top_k / n_experts))
        report(f"step {i}: loss {losses[-1]:.5f}, busiest expert {loads[-1]:.2f} of the mean")
    return losses, (loads[0], loads[-1])


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    losses, _ = train(tokens=a.tokens, steps=a.steps)
    sys.exit(0 if losses[-1] < losses[0] else 1)
