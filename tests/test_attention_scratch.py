"""Scratch of the attention half's module (no GPU needed): what a captured graph has the address of stays."""
import weakref

import torch

import paper_2602_11543_amd as S
from paper_2602_11543_amd.attention import DeviceAttention


def test_scratch_that_has_been_handed_out_stays():
    A = DeviceAttention.__new__(DeviceAttention)
    A.h, A.scratch = torch.empty(1), {}
    small, large = S.attn_shape(2, 128, 128, 4, 1, 64, S.SPES_BF16), S.attn_shape(2, 2, 6000, 4, 1, 64, S.SPES_BF16)
    first = A._scratch(small, 1)
    assert first.numel() >= S.spes_attn_scratch_bytes(small, 1) > 0
    held, at = weakref.ref(first), first.data_ptr()
    del first
    assert S.spes_attn_scratch_bytes(large, 0) > S.spes_attn_scratch_bytes(small, 1)
    second = A._scratch(large, 0)
    assert second.numel() >= S.spes_attn_scratch_bytes(large, 0)
    assert held() is not None and held().data_ptr() == at


def test_growing_scratch_is_bounded():
    """However slowly the need grows, all that is kept is a few times the largest."""
    A = DeviceAttention.__new__(DeviceAttention)
    A.h, A.scratch = torch.empty(1), {}
    kept, need = {}, 0
    for rows in range(1, 2000, 7):
        shape = S.attn_shape(1, rows, rows, 4, 1, 64, S.SPES_F32)
        need = max(need, S.spes_attn_scratch_bytes(shape, 1))
        t = A._scratch(shape, 1)
        assert t.numel() >= S.spes_attn_scratch_bytes(shape, 1)
        kept[t.data_ptr()] = t
    assert sum(t.numel() for t in kept.values()) <= 4 * need and len(kept) <= 24
