"""Routing where masks, biases, bad numbers and far logits meet: what counts for the choice, and gates that agree with it and with their gradient.

The choice is compared exactly with the definition in 64 bits, a masked expert left out first.  A score in 32 bits is within some 20 steps of
2^-24; sums c of a score and a bias that are nearer than 2^-18 of their size are drawn again.  Gates and gradients have K = 64 steps of their
terms, and half a step of its distance for every score that is e to the power of one."""
import math

import pytest
import torch

import paper_2602_11543_amd as S
from test_gpu_router import SIGMOID, forward

pytestmark = pytest.mark.gpu


def test_a_group_of_bad_numbers_does_not_open(device):
    """A NaN is passed over wherever it stands in its group: it does not stand in for a second score."""
    M, groups = 24, 3
    for at in range(8):
        for other in range(8):
            if other == at:
                continue
            logits = torch.full((1, M), -2.0, device="cuda")
            logits[0, at], logits[0, other] = math.nan, 3.0                 # 0.95 + 0.12
            logits[0, 8:16] = -4.0
            logits[0, 10], logits[0, 13] = 0.5, 0.4                         # 0.62 + 0.60, which wins
            idx, gate, _ = forward(logits, None, 3, S.router_opts(SIGMOID, groups, 1))
            assert idx.tolist() == [[10, 13, 8]], (at, other)
            assert bool(torch.isfinite(gate).all())
