"""The range of scales that attention takes (no GPU needed)."""
import ctypes

import paper_2602_11543_amd as S

LIB = ctypes.CDLL(S.library_path())
P = [0x10000 + 0x1000 * i for i in range(16)]          # aligned, never dereferenced
EINVAL = -1
vp = ctypes.c_void_p
LIB.spes_attn_fwd.argtypes, LIB.spes_attn_bwd.argtypes = [vp] * 11, [vp] * 15


def shape(scale, dtype, q_rows=64, k_rows=96):
    s = S.attn_shape(2, q_rows, k_rows, 4, 2, 64, dtype, 1, 0)
    s.scale = scale
    return s


def test_small_scales_of_bf16_gradients():
    """lse / scale has to be a number: 5 / 10^-38 is none in fp32."""
    for scale in (1e-45, 1e-38, 2.0 ** -121):
        s = shape(scale, S.SPES_BF16)
        assert LIB.spes_attn_bwd(ctypes.byref(s), *P[:13], None) == EINVAL and S.spes_attn_scratch_bytes(s, 1) == 0, scale
        assert S.spes_attn_scratch_bytes(s, 0) > 0 and S.spes_attn_scratch_bytes(shape(scale, S.SPES_F32), 1) > 0, scale
    assert S.spes_attn_scratch_bytes(shape(2.0 ** -120, S.SPES_BF16), 1) > 0


def test_large_scales():
    """Their scores would come of products that fp32 does not hold to 24 bits, and from 1.39 2^127 on scale log2 e is no number."""
    for scale in (3.4e38, 2.0 ** 127, 1.01 * 2.0 ** 95):
        for dtype in (S.SPES_BF16, S.SPES_F32):
            s = shape(scale, dtype)
            assert LIB.spes_attn_fwd(ctypes.byref(s), *P[:9], None) == EINVAL == LIB.spes_attn_bwd(ctypes.byref(s), *P[:13], None), scale
            assert S.spes_attn_scratch_bytes(s, 0) == 0 == S.spes_attn_scratch_bytes(s, 1), scale
    for backward in (0, 1):
        assert S.spes_attn_scratch_bytes(shape(2.0 ** 95, S.SPES_BF16), backward) > 0
