"""Attention forward and backward against the definition in 64 bits, element by element (allowances: attention_reference.py)."""
import math

import pytest
import torch

import paper_2602_11543_amd as S
from attention_reference import attention, excess

pytestmark = pytest.mark.gpu

SENTINEL = 7.0


def starts(lens, first=0):
    at = [first]
    for n in lens:
        at.append(at[-1] + n)
    return at


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Problem:
    """Tensors of one call.  gap: rows of no sequence ahead of the first and behind the last; room: rows of a sequence in a cache with k_len; layout: how the
    heads stand ('rows': side by side in a token; 'heads': a head's rows one behind the other; 'packed': views of one projection's output)."""

    def __init__(self, lens, keys=None, heads=2, kv=2, dim=64, dtype=torch.bfloat16, causal=True, window=0, gap=0, room=0, layout="rows", seed=0, scale=None,
                 size=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.keys = lens, list(lens) if keys is None else keys
        self.heads, self.kv, self.dim, self.dtype, self.causal, self.window = heads, kv, dim, dtype, causal, window
        self.scale = dim ** -0.5 if scale is None else scale
        q_at = starts(lens, gap)
        rows = q_at[-1] + gap
        if room:
            k_at = [gap + i * room for i in range(len(lens))]
            krows = gap + room * len(lens) + gap
            self.k_start, self.k_len = ints(k_at), ints(self.keys)
        else:
            k_at = starts(self.keys, gap)
            krows = k_at[-1] + gap
            self.k_start, self.k_len = ints(k_at), None
        self.q_start, self.rows, self.krows = ints(q_at), rows, krows
        self.seqs = [(q_at[i], n, k_at[i], m) for i, (n, m) in enumerate(zip(lens, self.keys))]

        def tensor(n, h):
            return (size * torch.randn(n, h, dim, generator=g)).to(dtype).cuda()

        q, k, v, self.d_o = tensor(rows, heads), tensor(krows, kv), tensor(krows, kv), (torch.randn(rows, heads, dim, generator=g)).to(dtype).cuda()
        # what stands in rows of no sequence must not matter
        mask = torch.ones(krows, dtype=torch.bool)
        for _, _, at, m in self.seqs:
            mask[at: at + m] = False
        k[mask], v[mask] = math.nan, math.nan
        mask = torch.ones(rows, dtype=torch.bool)
        mask[q_at[0]: q_at[-1]] = False
        q[mask], self.d_o[mask] = math.nan, math.inf
        self.layout = layout
        self.q, self.k, self.v = self._lay(q, "q"), self._lay(k, "k"), self._lay(v, "v")

    def _lay(self, t, name, fill=None):
        n, h, d = t.shape
        if self.layout == "rows":
            out = torch.empty_like(t)
        elif self.layout == "heads":
            out = torch.empty(h, n + 3, d, dtype=t.dtype, device=t.device)[:, 1: n + 1].transpose(0, 1)
        else:
            width = (self.heads + 2 * self.kv) * d
            at = {"q": 0, "k": self.heads * d, "v": (self.heads + self.kv) * d}[name]
            out = torch.empty(n, width, dtype=t.dtype, device=t.device)[:, at: at + h * d].view(n, h, d)
        out.copy_(t) if fill is None else out.fill_(fill)
        return out

    def shape(self):
        return S.attn_shape(len(self.lens), self.rows, self.krows, self.heads, self.kv, self.dim, S.SPES_F32 if self.dtype == torch.float32 else S.SPES_BF16,
                            int(self.causal), self.window, self.scale)

    def forward(self):
        o = torch.full((self.rows, self.heads, self.dim), SENTINEL, dtype=self.dtype, device="cuda")
        lse = torch.full((self.heads, self.rows), SENTINEL, device="cuda")
        scratch = torch.full((S.spes_attn_scratch_bytes(self.shape(), 0),), 255, dtype=torch.uint8, device="cuda")
        S.spes_attn_fwd(self.shape(), self.q, self.k, self.v, self.q_start, self.k_start, self.k_len, o, lse, scratch)
        return {"o": o, "lse": lse}

    def backward(self, o, lse):
        out = {"d" + n: self._lay(getattr(self, n), n, SENTINEL) for n in ("q", "k", "v")}
        scratch = torch.full((S.spes_attn_scratch_bytes(self.shape(), 1),), 255, dtype=torch.uint8, device="cuda")
        S.spes_attn_bwd(self.shape(), self.d_o, self.q, self.k, self.v, self.q_start, self.k_start, self.k_len, o, lse, *out.values(), scratch)
        return out

    def check(self, backward=True):
        print(self.lens, self.keys, self.heads, self.kv, self.dim, self.dtype, self.causal, self.window, self.layout, flush=True)
        got = self.forward()
        if backward:
            got.update(self.backward(**got))
        torch.cuda.synchronize()
        want = attention(self.q, self.k, self.v, self.seqs, self.scale, self.causal, self.window, self.d_o if backward else None)
        for name, (value, allow) in want.items():
            over, text = excess(got[name], value, allow)
            assert over <= 0, (name, over, text)
            outside = torch.isnan(value)                     # left as they were
            assert (got[name][outside] == SENTINEL).all(), name
        return got


BOTH = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("dim", [8, 40, 64, 72, 80, 128])
def test_widths(dtype, dim):
    Problem([130, 1, 65], heads=4, kv=2, dim=dim, dtype=dtype, seed=dim).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (4, 1), (6, 2), (5, 1), (7, 1), (12, 1), (64, 2), (130, 1)])
def test_shared_heads(dtype, heads, kv):
    Problem([1, 70, 33], heads=heads, kv=kv, dim=64, dtype=dtype, seed=heads).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("lens", [[1], [2], [31, 32, 33], [63], [64], [65], [127, 128, 129], [0, 5, 0, 0, 66, 0], [300], [1] * 70, [5] * 130])
def test_lengths(dtype, lens):
    Problem(lens, heads=4, kv=2, dim=64, dtype=dtype, seed=len(lens)).check()
    Problem(lens, heads=2, kv=2, dim=128, dtype=dtype, causal=False, seed=len(lens)).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("window", [1, 2, 17, 63, 64, 65, 100, 199, 200, 2 ** 31 - 1])
def test_windows(dtype, window):
    Problem([200, 3, 129], heads=4, kv=2, dim=64, dtype=dtype, window=window, seed=3).check()
    Problem([90, 3], keys=[200, 140], heads=3, kv=1, dim=128, dtype=dtype, window=window, seed=4).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,keys", [([5], [200]), ([130], [70]), ([200], [1]), ([64, 64], [65, 63]), ([10, 0, 20], [0, 40, 150]), ([1, 1, 1], [0, 1, 129]),
                                       ([3, 130], [0, 0])])
def test_queries_and_keys_of_unequal_number(dtype, causal, lens, keys):
    got = Problem(lens, keys, heads=4, kv=2, dim=64, dtype=dtype, causal=causal, seed=5).check()
    assert causal is False or torch.isinf(got["lse"]).any() == any(n > m for n, m in zip(lens, keys))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("layout", ["rows", "heads", "packed"])
def test_layouts_and_rows_of_no_sequence(dtype, layout):
    Problem([65, 129, 7], heads=4, kv=2, dim=80, dtype=dtype, gap=5, layout=layout, seed=6).check()
    if layout != "packed":
        Problem([3, 1, 7], keys=[100, 1, 64], heads=4, kv=2, dim=64, dtype=dtype, gap=5, room=131, layout=layout, seed=7).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("lens,keys,kw", [([1], [5000], {}), ([1, 1, 1], [3000, 1, 2049], dict(room=3001)), ([2, 3], [2500, 1999], dict(window=700)),
                                          ([4], [4096], dict(causal=False)), ([100], [1800], {}), ([1] * 9, [600] * 9, dict(room=640))])
def test_few_queries_against_a_long_cache(dtype, lens, keys, kw):
    p = Problem(lens, keys, heads=8, kv=2, dim=128, dtype=dtype, seed=8, **kw)
    p.check(backward=False)
    Problem(lens, keys, heads=3, kv=3, dim=64, dtype=dtype, seed=9, **kw).check()


def test_sequences_that_share_keys():
    """A common beginning, read by every sequence from one place of the cache."""
    p = Problem([1, 1, 1, 1], [700, 650, 1, 700], heads=4, kv=1, dim=64, room=700, seed=10)
    p.k_start = ints([0, 0, 0, 0])
    p.seqs = [(q0, lq, 0, lk) for q0, lq, _, lk in p.seqs]
    p.check(backward=False)


@pytest.mark.parametrize("dtype", BOTH)
def test_sharp_and_flat_scores(dtype):
    """Scores of some hundreds, and a scale that leaves them all alike."""
    Problem([150], heads=2, kv=1, dim=64, dtype=dtype, size=6.0, seed=11).check()
    Problem([150], heads=2, kv=1, dim=64, dtype=dtype, scale=1e-6, seed=12).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_rising_scores(dtype):
    """The maximum moves with every key, by little and by much."""
    for step in (0.05, 3.0):
        p = Problem([260], heads=1, kv=1, dim=64, dtype=dtype, causal=False, seed=13)
        p.q.fill_(0.5)
        p.k.copy_((step * torch.arange(260, device="cuda")[:, None, None] / 4).expand(260, 1, 64))
        p.check()


def test_descriptors_beyond_the_tensors_are_cut():
    """Rows that do not exist are no rows, whatever the descriptors say; nothing else is touched."""
    p = Problem([64, 64], heads=2, kv=2, dim=64, seed=14)
    for q_start, k_start, k_len, seqs in (([0, 64, 999], [0, 64, 999], None, p.seqs), ([-5, 64, 128], [-9, 64, 2 ** 31 - 1], None, p.seqs),
                                          ([0, 64, 128], [0, 64], [64, 2 ** 31 - 1], p.seqs), ([0, 64, 64], [0, 128, 64], None, [(0, 64, 0, 128)]),
                                          ([0, 64, 128], [0, 500], [64, 64], [(0, 64, 0, 64), (64, 64, 128, 0)]), ([0, 64, 128], [0, 64], [64, -3], [(0, 64, 0, 64), (64, 64, 64, 0)])):
        p.q_start, p.k_start, p.k_len, p.seqs = ints(q_start), ints(k_start), None if k_len is None else ints(k_len), seqs
        p.check(backward=False)


@pytest.mark.parametrize("dtype", BOTH)
def test_the_same_bits_every_time_and_everywhere(dtype):
    p = Problem([150, 150, 64], keys=[220, 220, 64], heads=8, kv=2, dim=64, dtype=dtype, causal=False, seed=15)
    q0, k0 = p.q[:150].clone(), p.k[:220].clone()
    p.q[150:300], p.k[220:440], p.v[220:440], p.d_o[150:300] = q0, k0, p.v[:220].clone(), p.d_o[:150].clone()
    p.q[7], p.d_o[7] = p.q[140].clone(), p.d_o[140].clone()          # copies within a sequence as well
    p.q[157], p.d_o[157] = p.q[140], p.d_o[140]
    a = p.forward()
    a.update(p.backward(**a))
    b = p.forward()
    b.update(p.backward(**b))
    for n in a:
        assert torch.equal(a[n], b[n]), n
    for n in ("o", "dq"):
        assert torch.equal(a[n][:150], a[n][150:300]) and torch.equal(a[n][7], a[n][140]), n
    for n in ("dk", "dv"):
        assert torch.equal(a[n][:220], a[n][220:440]), n


def test_gradients_against_differences():
    """Central differences of sum(o do) in fp32 storage along random directions.  With d = 2^-7: the forward's own error in the difference, at most
    2 x 2e-6 of the sum of |o do| over 2 d, and the third-order term of the difference, bounded by the difference at 2 d."""
    p = Problem([70, 33], heads=4, kv=2, dim=40, dtype=torch.float32, window=50, seed=16)
    f = p.forward()
    grads = p.backward(**f)

    def value(name, direction, d):
        t = getattr(p, name)
        keep = t.clone()
        t.add_(d * direction)
        o = p.forward()["o"]
        t.copy_(keep)
        return float((o.double() * p.d_o.double()).sum())

    g = torch.Generator(device="cuda").manual_seed(17)
    size = float((f["o"].double() * p.d_o.double()).abs().sum())
    for name in ("q", "k", "v"):
        t = getattr(p, name)
        direction = torch.randn(t.shape, device="cuda", generator=g)
        slope = float((grads["d" + name].double() * direction.double()).sum())
        d = 2.0 ** -7
        one = (value(name, direction, d) - value(name, direction, -d)) / (2 * d)
        two = (value(name, direction, 2 * d) - value(name, direction, -2 * d)) / (4 * d)
        noise = 4e-6 * size / (2 * d)
        # one - slope = c d^2, two - slope = 4 c d^2 up to higher orders: twice a third of their difference
        assert abs(one - slope) <= 2 * abs(two - one) / 3 + noise, (name, slope, one, two, noise)


def test_long_offsets():
    """Rows of a cache beyond 2^31 elements and 2^32 bytes."""
    rows, kv, dim = 2 ** 22 + 4096 + 100, 8, 128
    p = Problem([1, 1], [300, 257], heads=16, kv=kv, dim=dim, seed=18)
    k, v = (torch.empty(rows, kv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = [rows - 300, rows - 700]
    for (_, _, k0, lk), new in zip(p.seqs, at):
        k[new: new + lk], v[new: new + lk] = p.k[k0: k0 + lk], p.v[k0: k0 + lk]
    want = p.forward()
    p.k, p.v, p.krows, p.k_start, p.k_len = k, v, rows, ints(at), ints([300, 257])
    got = p.forward()
    ref = attention(p.q, k[at[1]:].contiguous(), v[at[1]:].contiguous(), [(q0, lq, new - at[1], lk) for (q0, lq, _, lk), new in zip(p.seqs, at)], p.scale, True, 0)
    for n in ("o", "lse"):
        assert excess(got[n], *ref[n])[0] <= 0 and excess(want[n], *ref[n])[0] <= 0, n


def test_another_stream_and_a_graph():
    """On a stream of its own, and captured: replays give the eager bits, with other inputs as well, beside eager calls that use other buffers."""
    p = Problem([100, 29], heads=4, kv=2, dim=64, seed=19)
    long = Problem([1, 2], [3000, 2000], heads=4, kv=2, dim=64, seed=20)

    def call(x):
        out = x.forward()
        out.update(x.backward(**out))
        return out

    side = torch.cuda.Stream()
    eager = [call(p), call(long)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = [call(p), call(long)]
    side.synchronize()
    for a, b in zip(eager, again):
        for n in a:
            assert torch.equal(a[n], b[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [call(p), call(long)]
    for i in range(3):
        p.q.mul_(1 + i / 4)
        long.k.mul_(0.5 + i / 4)
        graph.replay()
        eager = [call(p), call(long)]
        torch.cuda.synchronize()
        for a, b in zip(eager, captured):
            for n in a:
                assert torch.equal(a[n], b[n]), (i, n)


def test_nothing_to_do():
    for lens in ([], [0, 0]):
        p = Problem(lens, heads=2, kv=1, dim=64, gap=3)
        got = p.forward()
        got.update(p.backward(**got))
        torch.cuda.synchronize()
        for n, t in got.items():
            assert (t == SENTINEL).all(), n


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 32), (torch.bfloat16, 64), (torch.bfloat16, 96), (torch.bfloat16, 128), (torch.float32, 32), (torch.float32, 64),
                                       (torch.float32, 128)])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=100), dict(window=333, heads=3, kv=1), dict(heads=7, kv=1)])
def test_sequences_long_enough_for_two_sets_of_wavefronts(dtype, dim, kw):
    Problem([257, 640, 449], dtype=dtype, dim=dim, seed=dim, **kw).check()
    Problem([300, 290], keys=[600, 290], dtype=dtype, dim=dim, gap=3, layout="heads", seed=dim, **kw).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_many_blocks(dtype):
    """More than the chip holds at once, so one set of wavefronts to a block; sequences of unequal length."""
    lens = [1500, 3, 700, 64, 257, 1]
    Problem(lens, heads=32, kv=16, dim=64, dtype=dtype, seed=21).check()


@pytest.mark.parametrize("dim", [16, 32, 48, 56, 80, 96, 104, 112, 120])
@pytest.mark.parametrize("kw", [dict(lens=[150, 1, 70]), dict(lens=[90, 33], window=40, heads=3, kv=1, layout="packed"), dict(lens=[1, 2], keys=[700, 91], room=704, heads=6),
                                dict(lens=[700], keys=[900], causal=False)])
def test_widths_that_end_inside_a_fragment(dim, kw):
    Problem(**{**dict(dim=dim, dtype=torch.float32, seed=dim), **kw}).check()


@pytest.mark.parametrize("dim", [24, 64])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=90), dict(heads=80), dict(heads=120, window=200)])
def test_gradients_of_two_launches_with_two_sets_of_wavefronts(dim, kw):
    """More blocks than run at once, each launch's fewer."""
    Problem([300, 290], dim=dim, **{**dict(heads=40, kv=40, seed=dim), **kw}).check()


@pytest.mark.parametrize("dim", [72, 128])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=50), dict(heads=192)])
def test_gradients_of_long_heads_in_two_launches(dim, kw):
    lens = [1, 200, 64, 65, 129, 7, 90, 128, 33, 250, 12, 101, 64, 180, 5, 70]
    Problem(lens, dim=dim, **{**dict(heads=64, kv=64, seed=dim), **kw}).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("lens,keys", [([0, 0], [70, 33]), ([70, 33], [0, 0])])
def test_gradients_without_queries_or_keys(dtype, lens, keys):
    got = Problem(lens, keys=keys, dtype=dtype).check()
    assert all((got[n] == 0).all() for n in ("dq", "dk", "dv"))


@pytest.mark.parametrize("n,some", [(65, 3), (130, 1), (4097, 15), (4500, 17)])
def test_many_sequences_most_of_them_empty(n, some):
    lens = [0] * n
    for i in range(0, n, some):
        lens[i] = 1 + (7 * i) % 41
    lens[n // 2] = 300
    Problem(lens, heads=2, kv=1, dim=32, gap=5, seed=n).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_caches_in_any_order(dtype):
    for n in (5, 70):
        p = Problem([20 + i % 30 for i in range(n)], keys=[90] * n, room=97, heads=4, kv=2, gap=2, dtype=dtype, seed=n)
        order = torch.randperm(n, generator=torch.Generator().manual_seed(n)).tolist()
        p.k_start = p.k_start[order].contiguous()
        p.seqs = [(q, lq, p.seqs[o][2], m) for (q, lq, _, m), o in zip(p.seqs, order)]
        p.check()


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.bfloat16, 40), (torch.float32, 80)])
@pytest.mark.parametrize("n,kv", [(130, 8), (70, 16), (700, 8)])
def test_single_tokens_of_many_sequences(dtype, dim, n, kv):
    """Keys in parts of more than 64 sequences, and at 700 sequences whole, from more tiles than there are blocks."""
    Problem([i % 2 + (i % 7 == 0) for i in range(n)], keys=[(37 * i) % 300 for i in range(n)], room=300, heads=2 * kv, kv=kv, dim=dim, dtype=dtype, gap=1, seed=n).check(backward=False)
