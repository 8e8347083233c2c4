"""Attention at the ends of the range of scales, against the definition in 64 bits."""
import pytest
import torch

from test_gpu_attention import BOTH, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("size", [1.0, 2.0 ** 58])
def test_small_scales(dtype, size):
    """Scores that are all alike, and scores of some units from products of up to 2^123."""
    Problem([150, 1, 70], heads=2, kv=1, dim=64, dtype=dtype, scale=2.0 ** -120, size=size, seed=12).check()


def test_smaller_ones_where_nothing_is_divided_by_them():
    Problem([150], heads=2, kv=1, dim=64, dtype=torch.float32, scale=1e-38, seed=12).check()
    Problem([150], heads=2, kv=1, dim=64, scale=1e-38, seed=12).check(backward=False)


@pytest.mark.parametrize("dtype", BOTH)
def test_large_scales(dtype):
    Problem([150, 1, 70], heads=2, kv=1, dim=64, dtype=dtype, scale=2.0 ** 95, size=2.0 ** -49, seed=12).check()
