"""Micro-batches on a block: gradients are added to those of the batches before, from the first one on."""
import numpy as np
import pytest
import torch

from paper_2602_11543_amd.block import DeviceBlock

pytestmark = pytest.mark.gpu


def grads(b):
    return [b.d_norm_w, b.d_w_router, *b.grad.values()]


def test_accumulates_from_the_first_batch_on(device):
    T, d, M, f, k = 40, 64, 8, 32, 3
    mask = np.array([1, 0, 1, 1, 0, 0, 1, 0])
    new = lambda: DeviceBlock(T, d, M, f, k, mask, "f32", groups=4, kept_groups=3, seed=4)  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(5)
    batches = [[torch.randn(T, d, device="cuda", generator=g) for _ in range(3)] for _ in range(2)]
    alone = []
    for x, add, d_out in batches:
        b = new()
        b.forward(x, add)
        b.backward(d_out)
        alone.append([t.clone() for t in grads(b)])
    junk = torch.full((1 << 22,), float("nan"), device="cuda")          # what memory that is taken next may hold
    del junk
    b = new()
    for x, add, d_out in batches:
        b.forward(x, add)
        b.backward(d_out, accumulate=1)
    torch.cuda.synchronize()
    for got, one, two in zip(grads(b), *alone):
        assert torch.isfinite(got).all()
        # (one more addition in fp32, on sums whose last bits may fall another way)
        assert float((got - (one + two)).abs().max()) <= 8 * 2.0 ** -24 * float((one.abs() + two.abs()).max())
    x, add, d_out = batches[0]
    b.forward(x, add)
    b.backward(d_out)
    for got, one in zip(grads(b), alone[0]):
        assert torch.equal(got, one)
