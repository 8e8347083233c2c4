"""Refusals of the attention half of a block: bad arguments are rejected on the host, before any launch (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2602_11543_amd as S

LIB = ctypes.CDLL(S.library_path())
P = [0x10000 + 0x1000 * i for i in range(16)]          # aligned, never dereferenced
i32, vp, sz = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
EINVAL, ESHAPE, EALIGN = -1, -2, -3


def _qk(**over):
    s = S.qk_shape(8, 4, 2, 64, 64, S.SPES_BF16, 0, 100)
    for n, v in over.items():
        assert hasattr(s, n)
        setattr(s, n, v)
    return s


def _attn(**over):
    s = S.attn_shape(2, 64, 96, 4, 2, 64, S.SPES_BF16, 1, 0)
    for n, v in over.items():
        assert hasattr(s, n)
        setattr(s, n, v)
    return s


QK_EINVAL = [dict(T=-1), dict(heads=0), dict(kv_heads=0), dict(head_dim=0), dict(rot_dim=-16), dict(rot_dim=80), dict(dtype=2), dict(n_pos=-1), dict(eps=-1.0),
             dict(eps=float("nan")), dict(q_row=255), dict(k_row=127), dict(n_pos=0)]
QK_ESHAPE = [dict(head_dim=60, rot_dim=48, q_row=240, k_row=120), dict(head_dim=264, q_row=1056, k_row=528), dict(rot_dim=24), dict(T=2 ** 30)]
ATTN_EINVAL = [dict(n_seq=-1), dict(q_rows=-1), dict(k_rows=-1), dict(heads=0), dict(kv_heads=0), dict(head_dim=0), dict(dtype=5), dict(window=-1),
               dict(window=4, causal=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(kv_heads=3), dict(q_row=63),
               dict(q_head=0), dict(k_row=8), dict(k_head=-64), dict(v_row=0), dict(v_head=56)]
ATTN_ESHAPE = [dict(head_dim=60), dict(head_dim=136, q_row=544, q_head=136, k_row=272, k_head=136, v_row=272, v_head=136), dict(heads=2048, kv_heads=2048),
               dict(q_row=2 ** 20 + 8), dict(k_row=2 ** 20 + 8), dict(v_row=2 ** 20 + 8), dict(q_head=2 ** 27 + 8), dict(q_rows=2 ** 29),
               dict(n_seq=2 ** 30), dict(k_rows=2 ** 31 - 1, heads=1024, kv_heads=1024)]


def test_norm_and_rotation():
    fwd_, bwd_, bytes_ = LIB.spes_qk_rope_fwd, LIB.spes_qk_rope_bwd, LIB.spes_qk_rope_scratch_bytes
    fwd_.restype, fwd_.argtypes = i32, [vp] * 10
    bwd_.restype, bwd_.argtypes = i32, [vp] * 13 + [i32, vp, vp]
    bytes_.restype, bytes_.argtypes = sz, [vp]

    def fwd(shape=None, **over):
        a = {n: P[i] for i, n in enumerate(("q", "k", "qw", "kw", "table", "pos", "qo", "ko"))}
        a.update(over)
        s = shape if shape is not None else _qk()
        return fwd_(ctypes.byref(s) if s else None, *a.values(), None)

    def bwd(shape=None, **over):
        a = {n: P[i] for i, n in enumerate(("dq", "dk", "q", "k", "qw", "kw", "table", "pos", "dqi", "dki", "dqw", "dkw"))}
        scratch = over.pop("scratch", P[13])
        a.update(over)
        s = shape if shape is not None else _qk()
        return bwd_(ctypes.byref(s) if s else None, *a.values(), 0, scratch, None)

    for f in (fwd, bwd):
        assert f(False) == EINVAL
        for bad in QK_EINVAL:
            assert f(_qk(**bad)) == EINVAL, bad
        for bad in QK_ESHAPE:
            assert f(_qk(**bad)) == ESHAPE, bad
        for bad in (dict(q_row=260), dict(k_row=132), dict(dtype=0, q_row=258)):
            assert f(_qk(**bad)) == EALIGN, bad
        for bad in (dict(qw=None), dict(kw=None), dict(table=None)):
            assert f(**bad) == EINVAL, bad
        assert f(_qk(n_pos=7), pos=None) == EINVAL              # fewer positions than tokens
        assert f(_qk(rot_dim=0)) == EINVAL and f(_qk(rot_dim=0), table=None) == EINVAL      # nothing is rotated, yet a table or positions are given
    for n in ("q", "k", "qo", "ko"):
        assert fwd(**{n: None}) == EINVAL, n
    for n in ("q", "k", "qw", "kw", "table", "pos", "qo", "ko"):
        assert fwd(**{n: 0x10008}) == EALIGN, n
    for bad in (dict(dq=None), dict(dk=None), dict(q=None), dict(k=None), dict(dqi=None), dict(dki=None), dict(dqw=None), dict(dkw=None), dict(scratch=None),
                dict(qw=None, kw=None)):
        assert bwd(**bad) == EINVAL, bad
    for n in ("dq", "dk", "q", "k", "qw", "kw", "table", "pos", "dqi", "dki", "dqw", "dkw", "scratch"):
        assert bwd(**{n: 0x10008}) == EALIGN, n
    assert fwd(_qk(T=0), q=None, k=None, qo=None, ko=None) == 0
    assert bwd(_qk(T=0), dq=None, dk=None, q=None, k=None, dqi=None, dki=None, dqw=None, dkw=None, scratch=None) == 0
    for bad in QK_EINVAL[:-1] + QK_ESHAPE:
        assert bytes_(ctypes.byref(_qk(**bad))) == 0, bad
    assert bytes_(None) == 0 and bytes_(ctypes.byref(_qk())) > 0 and bytes_(ctypes.byref(_qk(T=0))) > 0


def test_attention():
    fwd_, bwd_, bytes_ = LIB.spes_attn_fwd, LIB.spes_attn_bwd, LIB.spes_attn_scratch_bytes
    fwd_.restype, fwd_.argtypes = i32, [vp] * 11
    bwd_.restype, bwd_.argtypes = i32, [vp] * 15
    bytes_.restype, bytes_.argtypes = sz, [vp, i32]

    def fwd(shape=None, **over):
        a = {n: P[i] for i, n in enumerate(("q", "k", "v", "qs", "ks", "kl", "o", "lse", "scratch"))}
        a.update(over)
        s = shape if shape is not None else _attn()
        return fwd_(ctypes.byref(s) if s else None, *a.values(), None)

    def bwd(shape=None, **over):
        a = {n: P[i] for i, n in enumerate(("do", "q", "k", "v", "qs", "ks", "kl", "o", "lse", "dq", "dk", "dv", "scratch"))}
        a.update(over)
        s = shape if shape is not None else _attn()
        return bwd_(ctypes.byref(s) if s else None, *a.values(), None)

    for f in (fwd, bwd):
        assert f(False) == EINVAL
        for bad in ATTN_EINVAL:
            assert f(_attn(**bad)) == EINVAL, bad
        for bad in ATTN_ESHAPE:
            assert f(_attn(**bad)) == ESHAPE, bad
        for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head"):
            assert f(_attn(**{n: 2052})) == EALIGN and f(_attn(dtype=0, **{n: 2050})) == EALIGN, n
        for n in ("q", "k", "v", "qs", "ks", "o", "lse", "scratch"):
            assert f(**{n: None}) == EINVAL, n
        for n in ("q", "k", "v", "o", "lse", "scratch"):
            assert f(**{n: 0x10008}) == EALIGN, n
        for n in ("qs", "ks", "kl"):
            assert f(**{n: 0x10002}) == EALIGN, n
        assert f(_attn(n_seq=0), q=None, k=None, v=None, qs=None, ks=None, o=None, lse=None, scratch=None) == 0
    for n in ("do", "dq", "dk", "dv"):
        assert bwd(**{n: None}) == EINVAL and bwd(**{n: 0x10008}) == EALIGN, n
    assert fwd(_attn(q_rows=0), q=None, o=None, lse=None) == 0 and bwd(_attn(q_rows=0, k_rows=0), q=None) == 0
    for bad in ATTN_EINVAL + ATTN_ESHAPE:
        assert bytes_(ctypes.byref(_attn(**bad)), 0) == 0 == bytes_(ctypes.byref(_attn(**bad)), 1), bad
    assert bytes_(None, 0) == 0 and bytes_(ctypes.byref(_attn()), 0) > 0 and bytes_(ctypes.byref(_attn()), 1) > 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    """(On the CPU no tensor fits; a wrong shape, type or layout is named before that.)"""
    s, q, k = _attn(), torch.zeros(64, 4, 64, dtype=torch.bfloat16), torch.zeros(96, 2, 64, dtype=torch.bfloat16)
    for args in ((q[:63], k, k), (q.float(), k, k), (q, k[:, :1], k), (q, k, k[..., :56]), (q, k, k)):
        with pytest.raises(S.SpesError):
            S.spes_attn_fwd(s, *args, None, None, None, None, None, None)
    p = _qk()
    x, y = torch.zeros(8, 4, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    for args in ((x[:7], y), (x, y.float()), (x.transpose(0, 1).contiguous().transpose(0, 1), y), (x, y)):
        with pytest.raises(S.SpesError):
            S.spes_qk_rope_fwd(p, *args, None, None, None, None, None, None)


def test_attention_limits_and_layouts_of_gradients():
    """More rows, keys or sequences than a launch has blocks for; gradients of which two elements would have one place."""
    fwd, bwd, need = LIB.spes_attn_fwd, LIB.spes_attn_bwd, LIB.spes_attn_scratch_bytes
    need.restype, need.argtypes = sz, [vp, i32]
    both = [dict(q_rows=2 ** 28 + 1), dict(n_seq=2 ** 21 + 1)]
    backward = [(dict(k_rows=2 ** 28 + 1), ESHAPE), (dict(q_row=64, q_head=64), EINVAL), (dict(q_row=248), EINVAL), (dict(k_row=64), EINVAL),
                (dict(k_head=128), EINVAL), (dict(v_row=120), EINVAL), (dict(v_row=64, v_head=64 * 95), EINVAL)]
    for bad in both:
        s = ctypes.byref(_attn(**bad))
        assert need(s, 0) == 0 == need(s, 1) and fwd(s, *P[:9], None) == ESHAPE == bwd(s, *P[:13], None), bad
    for bad, code in backward:
        s = ctypes.byref(_attn(**bad))
        assert need(s, 0) > 0 == need(s, 1) and bwd(s, *P[:13], None) == code, bad
    for good in (dict(), dict(q_row=264), dict(q_head=72, q_row=3 * 72 + 64), dict(k_row=64, k_head=96 * 64), dict(v_row=256, v_head=64), dict(q_rows=1, q_row=64),
                 dict(kv_heads=1, k_row=64, v_row=64)):
        assert need(ctypes.byref(_attn(**good)), 1) > 0, good


def test_norm_and_rotation_of_more_heads_than_are_numbered():
    """Kernels number a token's heads up to a few rounds behind the last one, and its elements, in 32 bits."""
    fwd, bwd, need = LIB.spes_qk_rope_fwd, LIB.spes_qk_rope_bwd, LIB.spes_qk_rope_scratch_bytes
    fwd.restype, fwd.argtypes = i32, [vp] * 10
    bwd.restype, bwd.argtypes = i32, [vp] * 13 + [i32, vp, vp]
    need.restype, need.argtypes = sz, [vp]
    for heads, kv in ((2 ** 31 - 2, 1), (2 ** 22, 1), (1, 2 ** 22), (2 ** 21 + 1, 2 ** 21)):
        s = S.qk_shape(1, 4, 2, 8, 0, S.SPES_BF16, 0, 0)
        s.heads, s.kv_heads, s.q_row, s.k_row = heads, kv, 8 * heads, 8 * kv
        r = ctypes.byref(s)
        assert fwd(r, *P[:4], None, None, *P[4:6], None) == ESHAPE == bwd(r, *P[:6], None, None, *P[6:10], 0, P[10], None) and need(r) == 0, (heads, kv)
    s.heads = s.kv_heads = 2 ** 21
    s.q_row = s.k_row = 2 ** 24
    assert need(ctypes.byref(s)) > 0
