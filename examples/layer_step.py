"""Trains one layer, attention and experts, on a fixed batch of documents of unequal length, and then takes single tokens through its attention.

    python examples/layer_step.py [--tokens 2048] [--steps 10]

The target is what another layer of the same shape makes of the batch; the loss is the mean square of the difference."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_11543_amd.attention import DeviceAttention  # noqa: E402
from paper_2602_11543_amd.block import DeviceBlock  # noqa: E402


class Layer:
    def __init__(self, tokens, d_model, heads, kv_heads, head_dim, n_experts, d_ff, top_k, mask, dtype, seed):
        self.attention = DeviceAttention(tokens, d_model, heads, kv_heads, head_dim, tokens, dtype, seed=seed)
        self.block = DeviceBlock(tokens, d_model, n_experts, d_ff, top_k, mask, dtype, seed=seed + 1)

    def forward(self, x, starts, pos):
        self.x, self.starts, self.pos = x, starts, pos
        return self.block.forward(x, self.attention.forward(x, starts, pos))

    def backward(self, d_out):
        d_sum = self.block.backward(d_out)
        return self.attention.backward(d_sum, self.x, self.starts, self.pos, d_sum)

    def step(self):
        self.attention.step()
        self.block.step()


def train(tokens=2048, d_model=256, heads=8, kv_heads=2, head_dim=64, n_experts=16, d_ff=128, top_k=2, steps=10, dtype="bf16", report=print):
    shape = dict(tokens=tokens, d_model=d_model, heads=heads, kv_heads=kv_heads, head_dim=head_dim, n_experts=n_experts, d_ff=d_ff, top_k=top_k, dtype=dtype)
    layer, teacher = Layer(mask=np.arange(n_experts) % 2, seed=1, **shape), Layer(mask=np.zeros(n_experts), seed=3, **shape)
    g = torch.Generator(device="cuda").manual_seed(5)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    # documents: a half, a quarter and so on of the batch, and what is left as one token each
    lens, left = [], tokens
    while left > 8:
        lens.append((left + 1) // 2)
        left -= lens[-1]
    lens += [1] * left
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n, device="cuda") for n in lens]).to(torch.int32)
    x = torch.randn(tokens, d_model, device="cuda", generator=g).to(t)
    target = teacher.forward(x, starts, pos).float()
    losses = []
    for i in range(steps):
        diff = layer.forward(x, starts, pos).float() - target
        layer.backward((2 / diff.numel() * 1024 * diff).to(t))          # (a loss scale: what the optimizer makes of the gradient does not depend on it)
        layer.step()
        losses.append(float(diff.square().mean()))
        report(f"step {i}: loss {losses[-1]:.5f}")
    # the first document once more, a token at a time
    attention, n = layer.attention, min(lens[0], 16)
    whole = attention.forward(x, starts, pos)[:n].float()
    attention.start_cache(1, lens[0])
    single = torch.cat([attention.decode(x[i: i + 1]) for i in range(n)]).float()
    report(f"one token at a time: {float((single - whole).norm() / whole.norm()):.4f} from the whole document in norm")
    return losses, single, whole


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    train(tokens=a.tokens, steps=a.steps)
