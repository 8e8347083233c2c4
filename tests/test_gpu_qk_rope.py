"""Norm and rotation of queries and keys: device kernels against the definition in 64 bits, element by element.

Allowances count roundings.  A sum over a head is sixteen terms one after the other and then four levels of a tree, so every statistic is within 24
steps of 2^-24 of its terms' magnitudes; K = 48 covers those and the operations on an element.  A result is rounded once, by at
most half a step of its type.  A weight's gradient sums n = T heads terms, each within K steps, in any order: n further steps bound it."""
import math

import pytest
import torch

import paper_2602_11543_amd as S

pytestmark = pytest.mark.gpu

K, STEP, SENTINEL = 48, 2.0 ** -24, 3.0
BOTH = [torch.bfloat16, torch.float32]


def turned(y, c, s, rot, interleaved):
    first = torch.arange(rot // 2, device=y.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else rot // 2)
    out = y.clone()
    out[..., first], out[..., second] = y[..., first] * c - y[..., second] * s, y[..., first] * s + y[..., second] * c
    return out


def magnitudes(y, c, s, rot, interleaved):
    """Of the terms of what is turned: |a c| + |b s| and |a s| + |b c|."""
    y, c, s = y.abs(), c.abs(), s.abs()
    return torch.maximum(turned(y, c, -s, rot, interleaved), turned(y, c, s, rot, interleaved))


def reference(x, w, table, pos, rot, interleaved, eps, dy):
    """{name: (value, magnitudes)} in 64 bits."""
    x, dy, n = x.double(), dy.double(), x.shape[0] * x.shape[1]
    c, s = torch.ones(1, 1, 0, device=x.device), torch.zeros(1, 1, 0, device=x.device)
    if rot:
        cs = table.double()[pos.long()][:, None]
        c, s = cs[..., : rot // 2], cs[..., rot // 2:]
    rstd = (x.square().mean(2, keepdim=True) + eps) ** -0.5 if w is not None else 1.0
    hat = x * rstd
    one = w.double() if w is not None else torch.ones(x.shape[2], dtype=torch.float64, device=x.device)
    y = hat * one
    out = {"y": (turned(y, c, s, rot, interleaved), magnitudes(y, c, s, rot, interleaved))}
    dz, mag = turned(dy, c, -s, rot, interleaved), magnitudes(dy, c, s, rot, interleaved)
    if w is None:
        out["dx"] = (dz, mag)
        return out
    h, hm = dz * one, mag * one.abs()
    out["dx"] = (rstd * (h - hat * (h * hat).mean(2, keepdim=True)), rstd * (hm + hat.abs() * (hm * hat.abs()).mean(2, keepdim=True)))
    out["dw"] = ((dz * hat).sum((0, 1)), (mag * hat.abs()).sum((0, 1)) * (1 + n / K))
    return out


def within(got, want, what):
    value, mag = want
    u = torch.finfo(got.dtype).eps / 2 if got.dtype == torch.bfloat16 else 0.0
    assert torch.isfinite(got).all(), what
    over = (got.double() - value).abs() - u * (1 + 2.0 ** -6) * value.abs() - K * STEP * (mag + value.abs()) - 2.0 ** -126
    assert float(over.max()) <= 0, (what, float(over.max()), float((got.double() - value).abs().max()))


class Problem:
    def __init__(self, T, heads=4, kv=2, dim=64, rot=None, interleaved=False, dtype=torch.bfloat16, norm=True, packed=True, n_pos=500, pos="some", seed=0):
        g = torch.Generator().manual_seed(seed)
        rot = dim // 16 * 16 if rot is None else rot
        self.T, self.heads, self.kv, self.dim, self.rot, self.interleaved, self.dtype = T, heads, kv, dim, rot, interleaved, dtype
        n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.width = (heads + 2 * kv) * dim
        self.qkv = (n(T, self.width) * (0.2 + n(T, 1).abs())).to(dtype).cuda()
        if packed:
            self.q, self.k = self.views(self.qkv)
        else:
            self.q, self.k = (t.contiguous() for t in self.views(self.qkv))
        self.packed = packed
        self.qw, self.kw = ((1 + 0.3 * n(dim)).to(dtype).cuda() for _ in range(2)) if norm else (None, None)
        self.dq, self.dk = n(T, heads, dim).to(dtype).cuda(), n(T, kv, dim).to(dtype).cuda()
        self.n_pos = max(n_pos, T) if pos == "none" else n_pos
        angle = torch.arange(self.n_pos).double()[:, None] * 10000.0 ** (-2.0 / max(rot, 1) * torch.arange(rot // 2).double())
        self.table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda() if rot else None
        self.pos = torch.randint(0, self.n_pos, (T,), generator=g).to(torch.int32).cuda() if rot and pos == "some" else None
        self.eps = 1e-6

    def views(self, t):
        H, Kv, D = self.heads, self.kv, self.dim
        return t[:, : H * D].view(-1, H, D), t[:, H * D: (H + Kv) * D].view(-1, Kv, D)

    def shape(self):
        return S.qk_shape(self.T, self.heads, self.kv, self.dim, self.rot, S.SPES_F32 if self.dtype == torch.float32 else S.SPES_BF16, int(self.interleaved),
                          self.n_pos, self.eps)

    def forward(self):
        q, k = (torch.full(t.shape, SENTINEL, dtype=self.dtype, device="cuda") for t in (self.dq, self.dk))
        S.spes_qk_rope_fwd(self.shape(), self.q, self.k, self.qw, self.kw, self.table, self.pos, q, k)
        return q, k

    def backward(self, accumulate=None, frozen=False):
        grad = torch.full_like(self.qkv, SENTINEL)
        dq, dk = self.views(grad)
        if not self.packed:
            dq, dk = dq.contiguous(), dk.contiguous()
        dw = [None, None]
        if self.qw is not None and not frozen:
            dw = [torch.full((self.dim,), math.nan, device="cuda") if accumulate is None else accumulate[i].clone() for i in range(2)]
        scratch = torch.full((S.spes_qk_rope_scratch_bytes(self.shape()),), 255, dtype=torch.uint8, device="cuda")
        S.spes_qk_rope_bwd(self.shape(), self.dq, self.dk, self.q, self.k, self.qw, self.kw, self.table, self.pos, dq, dk, *dw, int(accumulate is not None),
                           None if dw[0] is None else scratch)
        if self.packed:                 # the values' part is not this call's
            assert (grad[:, (self.heads + self.kv) * self.dim:] == SENTINEL).all()
        return dq, dk, dw

    def check(self):
        print(self.T, self.heads, self.kv, self.dim, self.rot, self.interleaved, self.dtype, flush=True)
        pos = torch.arange(self.T, device="cuda") if self.pos is None else self.pos
        y, (dq, dk, dw) = self.forward(), self.backward()
        for i, (x, w, dy, dx) in enumerate(((self.q, self.qw, self.dq, dq), (self.k, self.kw, self.dk, dk))):
            want = reference(x, w, self.table, pos, self.rot, self.interleaved, self.eps, dy)
            if self.T:
                within(y[i], want["y"], ("y", i))
                within(dx, want["dx"], ("dx", i))
            if w is not None:
                within(dw[i], want["dw"], ("dw", i))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(8, 0), (16, 16), (24, 16), (32, 16), (40, 32), (64, 64), (72, 64), (80, 48), (96, 96), (120, 16), (128, 128), (128, 0),
                                     (160, 160), (248, 16), (256, 256), (256, 240), (256, 16)])
def test_widths(dtype, interleaved, dim, rot):
    Problem(37, dim=dim, rot=rot, interleaved=interleaved, dtype=dtype, seed=dim + rot).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("T,heads,kv", [(0, 2, 1), (1, 1, 1), (1, 5, 5), (2, 3, 1), (255, 12, 12), (1000, 7, 3), (5000, 8, 2), (3, 200, 1)])
def test_tokens_and_heads(dtype, T, heads, kv):
    Problem(T, heads=heads, kv=kv, dim=64, dtype=dtype, seed=T).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("kw", [dict(norm=False), dict(norm=False, rot=0), dict(packed=False), dict(pos="none"), dict(norm=False, packed=False, interleaved=True)])
def test_forms(dtype, kw):
    Problem(133, dim=80, dtype=dtype, seed=1, **kw).check()


def test_without_a_norm_the_inputs_are_not_needed():
    p = Problem(50, dtype=torch.float32, norm=False, seed=2)
    want = p.backward()
    p.q = p.k = None
    got = p.backward()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", BOTH)
def test_gradients_of_weights_accumulate_and_may_be_left_out(dtype):
    p = Problem(300, dtype=dtype, seed=3)
    dq, dk, dw = p.backward()
    start = [torch.randn(p.dim, device="cuda") for _ in range(2)]
    more = p.backward(accumulate=start)
    for a, b, c in zip(start, dw, more[2]):
        assert torch.equal(a + b, c)
    frozen = p.backward(frozen=True)
    assert torch.equal(frozen[0], dq) and torch.equal(frozen[1], dk) and frozen[2] == [None, None]
    empty = Problem(0, dtype=dtype)
    kept = empty.backward(accumulate=start)[2]
    assert all(torch.equal(a, b) for a, b in zip(start, kept)) and all((t == 0).all() for t in empty.backward()[2])


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_position_that_the_table_does_not_have(interleaved):
    p = Problem(9, dim=80, rot=32, interleaved=interleaved, dtype=torch.float32, n_pos=20, seed=4)
    want = p.forward()
    p.pos[2], p.pos[5], p.pos[7] = 20, -1, 2 ** 31 - 1
    got = p.forward()
    for a, b in zip(got, want):
        for t in range(9):
            if t in (2, 5, 7):
                assert torch.isnan(a[t, :, :32]).all() and torch.equal(a[t, :, 32:], b[t, :, 32:])
            else:
                assert torch.equal(a[t], b[t])


@pytest.mark.parametrize("dtype", BOTH)
def test_zeros_and_extremes(dtype):
    """A head of zeros is zeros and has a finite gradient; large and small values keep their direction."""
    p = Problem(6, dtype=dtype, seed=5)
    p.qkv[0] = 0
    p.qkv[1] *= 1e15
    p.qkv[2] *= 1e-12
    p.check()
    assert (p.forward()[0][0] == 0).all()


@pytest.mark.parametrize("dtype", BOTH)
def test_the_same_bits_every_time_and_everywhere(dtype):
    p = Problem(400, heads=8, kv=8, dim=128, dtype=dtype, seed=6)
    p.kw.copy_(p.qw)
    p.qkv[300] = p.qkv[3]
    p.dq[300], p.dk[300], p.pos[300] = p.dq[3].clone(), p.dk[3].clone(), p.pos[3].clone()
    p.qkv[5, 8 * 128: 16 * 128] = p.qkv[5, : 8 * 128]           # a key that is a query
    a, b, ga, gb = p.forward(), p.forward(), p.backward(), p.backward()
    for x, y in zip((*a, *ga[:2], *ga[2]), (*b, *gb[:2], *gb[2])):
        assert torch.equal(x, y)
    for x in (*a, *ga[:2]):
        assert torch.equal(x[3], x[300])
    assert torch.equal(a[0][5], a[1][5])


def test_gradients_against_differences():
    """Central differences in fp32 storage: at d = 2^-7 the forward's error is at most 2^-21 of the sum of magnitudes over 2 d; the third-order term is a
    third of the difference to 2 d, twice over."""
    p = Problem(40, heads=3, kv=2, dim=40, rot=32, dtype=torch.float32, seed=7)
    dq, dk, dw = p.backward()
    g = torch.Generator(device="cuda").manual_seed(8)
    for i, (x, dx, w, dy) in enumerate(((p.q, dq, p.qw, p.dq), (p.k, dk, p.kw, p.dk))):
        size = float((p.forward()[i].double() * dy.double()).abs().sum())
        for t, grad in ((x, dx), (w, dw[i])):
            direction = torch.randn(t.shape, device="cuda", generator=g) * 0.1

            def value(d):
                keep = t.clone()
                t.add_(d * direction)
                y = float((p.forward()[i].double() * dy.double()).sum())
                t.copy_(keep)
                return y

            d = 2.0 ** -7
            one, two = (value(d) - value(-d)) / (2 * d), (value(2 * d) - value(-2 * d)) / (4 * d)
            slope = float((grad.double() * direction.double()).sum())
            assert abs(one - slope) <= 2 * abs(two - one) / 3 + 2.0 ** -21 * size / (2 * d), (i, one, two, slope)


def test_another_stream_and_a_graph():
    p = Problem(500, seed=9)

    def call():
        dq, dk, dw = p.backward()
        return (*p.forward(), dq, dk, *dw)

    eager = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, again))
    views = p.views(torch.full_like(p.qkv, SENTINEL))
    assert views[0].shape == eager[2].shape
    q, k = (torch.empty_like(t) for t in eager[:2])
    grad, dw = torch.empty_like(p.qkv), [torch.empty(p.dim, device="cuda") for _ in range(2)]
    scratch = torch.empty(S.spes_qk_rope_scratch_bytes(p.shape()), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.spes_qk_rope_fwd(p.shape(), p.q, p.k, p.qw, p.kw, p.table, p.pos, q, k)
        S.spes_qk_rope_bwd(p.shape(), p.dq, p.dk, p.q, p.k, p.qw, p.kw, p.table, p.pos, *p.views(grad), *dw, 0, scratch)
    for i in range(3):
        p.qkv.mul_(1.25)
        p.pos.copy_((p.pos + 7) % p.n_pos)
        graph.replay()
        eager = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (q, k, *p.views(grad), *dw))), i


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("kw", [dict(heads=16, kv=4, dim=128), dict(heads=5, kv=3, dim=64, interleaved=True), dict(heads=9, kv=9, dim=256, rot=64), dict(heads=30, kv=1, dim=64, norm=False)])
def test_tensors_that_the_caches_do_not_hold(dtype, kw):
    """More than 256 MB pass; the kernels for that take whole tokens."""
    size = 4 if dtype == torch.float32 else 2
    T = 300 * 2 ** 20 // (2 * size * (kw["heads"] + kw["kv"]) * kw["dim"]) + 3
    p = Problem(T, dtype=dtype, seed=10, **kw)
    p.check()
    start = [torch.randn(p.dim, device="cuda") for _ in range(2)]
    if p.qw is not None:
        for a, b, c in zip(start, p.backward()[2], p.backward(accumulate=start)[2]):
            assert torch.equal(a + b, c)
    p.pos[T - 2] = -1
    assert torch.isnan(p.forward()[1][T - 2, :, : p.rot]).all()


def test_a_missing_position_stays_with_its_token():
    """The gradients of the other tokens are what they were; those of the token and the weights' are NaN."""
    for T in (50, 300 * 2 ** 20 // (2 * 2 * 4 * 64)):
        p = Problem(T, heads=3, kv=1, dim=64, seed=11)
        want = p.backward()
        p.pos[7] = 10 ** 6
        got = p.backward()
        keep = torch.arange(T, device="cuda") != 7
        for a, b in zip(got[:2], want[:2]):
            assert torch.equal(a[keep], b[keep]) and torch.isnan(a[7]).all()
        assert all(torch.isnan(w).all() for w in got[2])
