"""Refusals of the operators around the expert layer: bad arguments are rejected on the host, before any launch (no GPU needed)."""
import ctypes

import paper_2602_11543_amd as S

LIB = ctypes.CDLL(S.library_path())
P = [0x10000 + 0x1000 * i for i in range(16)]          # aligned, never dereferenced
i32, i64, vp, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
EINVAL, ESHAPE, EALIGN = -1, -2, -3


def test_norm_forward():
    fn = LIB.spes_norm_fwd
    fn.restype, fn.argtypes = i32, [i32] * 4 + [vp, i64, vp, i64, vp, vp, f32] + [vp] * 5

    def fwd(kind=0, rows=4, cols=64, dtype=1, x=P[0], xs=64, add=None, as_=0, w=P[1], b=P[2], eps=1e-5, sum_=None, y=P[3], mean=P[4], rstd=P[5]):
        return fn(kind, rows, cols, dtype, x, xs, add, as_, w, b, eps, sum_, y, mean, rstd, None)

    for bad in (dict(kind=2), dict(rows=-1), dict(cols=0), dict(dtype=2), dict(x=None), dict(xs=63), dict(w=None), dict(y=None), dict(rstd=None),
                dict(mean=None), dict(kind=1), dict(add=P[6], as_=64), dict(add=P[6], as_=63, sum_=P[7]), dict(sum_=P[7]), dict(eps=-1.0),
                dict(eps=float("nan"))):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(cols=16385, xs=16385) == ESHAPE
    for bad in (dict(x=P[0] + 1), dict(dtype=0, x=P[0] + 2), dict(w=P[1] + 8), dict(b=P[2] + 2), dict(y=P[3] + 4), dict(mean=P[4] + 4),
                dict(rstd=P[5] + 4), dict(add=P[6] + 1, as_=64, sum_=P[7]), dict(add=P[6], as_=64, sum_=P[7] + 2)):
        assert fwd(**bad) == EALIGN, bad
    assert fwd(rows=0, x=None, w=None) == 0            # nothing to do


def test_norm_backward():
    fn = LIB.spes_norm_bwd
    fn.restype, fn.argtypes = i32, [i32] * 4 + [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, i32, vp, vp]

    def bwd(kind=0, rows=4, cols=64, dtype=1, dy=P[0], gs=64, x=P[1], xs=64, w=P[2], mean=P[3], rstd=P[4], dres=None, rs=0, dx=P[5], dw=P[6], db=P[7],
            scratch=P[8]):
        return fn(kind, rows, cols, dtype, dy, gs, x, xs, w, mean, rstd, dres, rs, dx, dw, db, 0, scratch, None)

    for bad in (dict(kind=-1), dict(rows=-1), dict(cols=0), dict(dtype=7), dict(dy=None), dict(gs=10), dict(x=None), dict(xs=63), dict(w=None), dict(mean=None),
                dict(kind=1), dict(rstd=None), dict(dx=None), dict(dres=P[9], rs=63), dict(dw=None), dict(scratch=None)):
        assert bwd(**bad) == EINVAL, bad
    assert bwd(cols=20000, gs=20000, xs=20000) == ESHAPE
    for bad in (dict(dy=P[0] + 1), dict(x=P[1] + 1), dict(w=P[2] + 2), dict(dx=P[5] + 2), dict(dw=P[6] + 4), dict(db=P[7] + 4), dict(scratch=P[8] + 4),
                dict(dres=P[9] + 1, rs=64)):
        assert bwd(**bad) == EALIGN, bad
    assert bwd(rows=0, dw=None, db=None, scratch=None) == 0
    assert S.spes_norm_scratch_bytes(100, 0) == 0 and S.spes_norm_scratch_bytes(-1, 64) == 0 and S.spes_norm_scratch_bytes(100, 16385) == 0
    assert S.spes_norm_scratch_bytes(0, 64) > 0


def test_router():
    fwd_, bwd_ = LIB.spes_router_fwd, LIB.spes_router_bwd
    fwd_.restype, fwd_.argtypes = i32, [i32, i32, i32, vp] + [vp] * 6
    bwd_.restype, bwd_.argtypes = i32, [i32, i32, i32, vp] + [vp] * 5

    def opts(o):
        return None if o is None else ctypes.byref(S.router_opts(*o))

    def fwd(T=8, M=64, k=8, o=(0, 1, 1, 1, 1.0), logits=P[0], bias=None, idx=P[1], gate=P[2], count=P[3]):
        return fwd_(T, M, k, opts(o), logits, bias, idx, gate, count, None)

    def bwd(T=8, M=64, k=8, o=(0, 1, 1, 1, 1.0), logits=P[0], idx=P[1], dgate=P[2], dlogits=P[3]):
        return bwd_(T, M, k, opts(o), logits, idx, dgate, dlogits, None)

    shapes = (dict(T=-1), dict(M=0), dict(k=0), dict(k=65), dict(o=None), dict(o=(2, 1, 1, 1, 1.0)), dict(o=(0, 0, 1, 1, 1.0)), dict(o=(0, 8, 0, 1, 1.0)),
              dict(o=(0, 8, 9, 1, 1.0)), dict(o=(0, 7, 3, 1, 1.0)), dict(o=(0, 16, 1, 1, 1.0)), dict(o=(0, 1, 1, 1, float("inf"))), dict(o=(0, 1, 1, 1, float("nan"))))
    for bad in shapes + (dict(logits=None), dict(idx=None), dict(gate=None), dict(count=None)):
        assert fwd(**bad) == EINVAL, bad
    for bad in shapes + (dict(logits=None), dict(idx=None), dict(dgate=None), dict(dlogits=None)):
        assert bwd(**bad) == EINVAL, bad
    for f in (fwd, bwd):
        assert f(M=513) == ESHAPE and f(k=17) == ESHAPE and f(o=(0, 32, 32, 1, 1.0)) == ESHAPE
    for bad in (dict(logits=P[0] + 4), dict(bias=P[5] + 4), dict(idx=P[1] + 4), dict(gate=P[2] + 8), dict(count=P[3] + 4)):
        assert fwd(**bad) == EALIGN, bad
    for bad in (dict(logits=P[0] + 4), dict(idx=P[1] + 4), dict(dgate=P[2] + 8), dict(dlogits=P[3] + 4)):
        assert bwd(**bad) == EALIGN, bad
    assert bwd(T=0, logits=None, idx=None, dgate=None, dlogits=None) == 0


def test_orthogonalize_and_muon():
    fn, mu = LIB.spes_orthogonalize, LIB.spes_masked_muon
    fn.restype, fn.argtypes = i32, [i32] * 4 + [vp, vp, i32, vp, vp, vp]
    mu.restype, mu.argtypes = i32, [i32] * 4 + [vp] * 5 + [f32, f32, i32, f32, f32, i32, vp, f32, vp, vp]
    c3 = lambda *v: (f32 * 3)(*v)  # noqa: E731

    def orth(n=2, rows=64, cols=32, dtype=1, src=P[0], out=P[1], steps=5, coef=None, scratch=P[2]):
        return fn(n, rows, cols, dtype, src, out, steps, coef, scratch, None)

    for bad in (dict(n=0), dict(rows=0), dict(cols=-1), dict(dtype=2), dict(src=None), dict(out=None), dict(scratch=None), dict(steps=0), dict(steps=65),
                dict(coef=c3(1, float("nan"), 0))):
        assert orth(**bad) == EINVAL, bad
    for bad in (dict(rows=16385), dict(cols=16385), dict(n=65536), dict(n=60000, rows=16384, cols=16384)):
        assert orth(**bad) == ESHAPE, bad
    for bad in (dict(src=P[0] + 8), dict(out=P[1] + 2), dict(scratch=P[2] + 4)):
        assert orth(**bad) == EALIGN, bad

    mask = (ctypes.c_uint8 * 3)(1, 0, 1)
    none = (ctypes.c_uint8 * 3)(0, 0, 0)

    def muon(E=3, rows=64, cols=32, dtype=1, param=P[0], mask=mask, master=P[1], m=P[2], grad=P[3], beta=0.95, steps=5, coef=None, scratch=P[4]):
        return mu(E, rows, cols, dtype, param, mask, master, m, grad, 0.1, beta, 1, 0.1, 1.0, steps, coef, 1.0, scratch, None)

    for bad in (dict(E=0), dict(rows=0), dict(dtype=9), dict(param=None), dict(mask=None), dict(master=None), dict(m=None), dict(grad=None), dict(beta=1.0),
                dict(beta=-0.1), dict(steps=0), dict(scratch=None), dict(coef=c3(float("inf"), 0, 0))):
        assert muon(**bad) == EINVAL, bad
    assert muon(rows=20000) == ESHAPE
    for bad in (dict(param=P[0] + 8), dict(master=P[1] + 4), dict(m=P[2] + 4), dict(grad=P[3] + 4), dict(scratch=P[4] + 4)):
        assert muon(**bad) == EALIGN, bad
    assert muon(mask=none, master=None, m=None, grad=None, scratch=None) == 0
    assert S.spes_orthogonalize_scratch_bytes(0, 8, 8, 0) == 0 and S.spes_orthogonalize_scratch_bytes(1, 8, 20000, 0) == 0
    assert S.spes_orthogonalize_scratch_bytes(2, 64, 96, 0) > S.spes_orthogonalize_scratch_bytes(2, 64, 96, 1) > 0


def test_layer_behind_a_given_routing():
    fwd_, bwd_ = LIB.spes_moe_fwd_routed, LIB.spes_moe_bwd_routed
    fwd_.restype, fwd_.argtypes = i32, [vp] * 11
    bwd_.restype, bwd_.argtypes = i32, [vp] * 13 + [i32, vp]
    shape = S.moe_shape(64, 64, 8, 64, 2, S.SPES_BF16, 0)
    mask = (ctypes.c_uint8 * 8)(1)

    def fwd(sh=shape, **over):
        a = {n: P[i] for i, n in enumerate(("x", "idx", "gate", "wg", "wu", "wd", "y", "count", "ctx"))}
        a.update(over)
        return fwd_(ctypes.byref(sh), *a.values(), None)

    def bwd(sh=shape, **over):
        a = dict(dy=P[0], x=P[1], wg=P[2], wu=P[3], wd=P[4], ctx=P[5], mask=ctypes.cast(mask, vp), dx=P[6], dgate=P[7], dg=P[8], du=P[9], dd=P[10])
        a.update(over)
        return bwd_(ctypes.byref(sh), *a.values(), 0, None)

    for n in ("x", "idx", "gate", "wg", "wu", "wd", "y", "count", "ctx"):
        assert fwd(**{n: None}) == EINVAL and fwd(**{n: 0x10008}) == EALIGN, n
    for n in ("dy", "x", "wg", "wu", "wd", "ctx", "mask", "dx", "dgate", "dg"):
        assert bwd(**{n: None}) == EINVAL, n
    for n in ("dy", "x", "wg", "wu", "wd", "ctx", "dx", "dgate", "dg", "du", "dd"):
        assert bwd(**{n: 0x10008}) == EALIGN, n
    for f in (fwd, bwd):
        assert f(S.moe_shape(64, 64, 8, 64, 9, 1, 0)) == EINVAL and f(S.moe_shape(64, 64, 128, 64, 2, 1, 0)) == ESHAPE
