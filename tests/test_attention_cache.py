"""Caches of the attention half's module (no GPU needed)."""
import pytest
import torch

import paper_2602_11543_amd as S
from paper_2602_11543_amd.attention import DeviceAttention


@pytest.mark.parametrize("n_seq,room", [(2 ** 20, 2 ** 20), (3, 2 ** 31 - 1), (2 ** 16, 2 ** 15), (1, 2 ** 40), (-1, 8), (8, -1)])
def test_caches_of_more_rows_than_are_numbered(n_seq, room):
    """Rows are numbered in 32 bits; nothing is allocated for such a cache, and what was there stays."""
    A = DeviceAttention.__new__(DeviceAttention)
    A.h, A.dt, A.K, A.D, A.n_pos, A.cache, A.taken = torch.empty(1), S.SPES_F32, 1, 8, 100, None, 7
    with pytest.raises(S.SpesError):
        A.start_cache(n_seq, room)
    assert A.cache is None and A.taken == 7
    A.start_cache(2, 3)
    assert A.cache[0].shape == (2, 3, 1, 8) and A.row0.tolist() == [0, 3] and A.spare.tolist() == [6, 6] and A.limit == 3
