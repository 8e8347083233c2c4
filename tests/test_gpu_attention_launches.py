"""Gradients at the most sequences that a launch takes, where those of queries and of keys are launches of their own in fp32 as well."""
import pytest
import torch

import paper_2602_11543_amd as S
from test_gpu_attention import Problem

pytestmark = pytest.mark.gpu


class Scattered(Problem):
    """Few sequences among 2^22 places, the others empty."""

    def __init__(self, lens, **kw):
        super().__init__(lens, **kw)
        self.places = 2 ** 22 // self.kv
        at = [0, 1, 4097, self.places // 2 + 65, self.places - 2, self.places - 1]
        for name, n in (("q_start", self.lens), ("k_start", self.keys)):
            count = torch.zeros(self.places + 1, dtype=torch.int32)
            count[[i + 1 for i in at]] = torch.tensor(n, dtype=torch.int32)
            setattr(self, name, count.cumsum(0).to(torch.int32).cuda())

    def shape(self):
        s = super().shape()
        if hasattr(self, "places"):
            s.n_seq = self.places
        return s


@pytest.mark.parametrize("dim", [24, 48, 64, 72, 88, 104, 128])
def test_launches_of_their_own(dim):
    """2^23 blocks and more."""
    Scattered([70, 1, 130, 33, 64, 90], heads=2, kv=1, dim=dim, dtype=torch.float32, seed=dim).check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_as_many_places_of_shared_heads(dtype):
    Scattered([70, 1, 130, 33, 64, 90], keys=[80, 5, 0, 300, 64, 100], heads=4, kv=4, dim=40, dtype=dtype, causal=False, seed=1).check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [40, 80, 128])
@pytest.mark.parametrize("lens,times", [([128, 128], 160), ([70, 1, 130, 33], 100), ([1100, 900], 6)])
def test_gradients_are_the_same_in_one_launch_and_in_two(dtype, dim, lens, times):
    """A batch whose blocks run as one launch, and many of it in one batch, whose blocks do or do not."""
    few = Problem(lens, heads=8, kv=4, dim=dim, dtype=dtype, seed=dim)
    many = Problem(lens * times, heads=8, kv=4, dim=dim, dtype=dtype, seed=dim)
    for name in ("q", "k", "v", "d_o"):
        getattr(many, name).copy_(getattr(few, name).repeat(times, 1, 1))
    f = few.forward()             # (of both: the forward of few blocks has its keys' sums in two sets)
    want, got = few.backward(**f), many.backward(f["o"].repeat(times, 1, 1), f["lse"].repeat(1, times))
    for name in ("dq", "dk", "dv"):
        assert torch.equal(got[name], want[name].repeat(times, 1, 1)), name
