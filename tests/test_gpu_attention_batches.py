"""The attention half of a block over the batches and tokens of a longer run: batches that do not fill its rows, graphs beside eager calls, caches that fill up."""
import pytest
import torch

import paper_2602_11543_amd as S
from paper_2602_11543_amd.attention import DeviceAttention
from test_gpu_attention_block import TOL16, TOL32, far

pytestmark = pytest.mark.gpu

D_MODEL = 64


def make(T, dtype="bf16", seed=1, **kw):
    A = DeviceAttention(T, D_MODEL, **{**dict(heads=4, kv_heads=2, head_dim=32, n_pos=128, dtype=dtype, seed=seed), **kw})
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    for n in ("norm", "q", "k"):
        A.w[n].copy_(1 + 0.2 * torch.randn(A.w[n].shape, device="cuda", generator=g))
    return A


def batch(A, starts, T=None, seed=2):
    """x, d_add, starts, pos of T rows, the rows of no sequence among them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = A.T if T is None else T
    x, d_add = (torch.randn(T, D_MODEL, device="cuda", generator=g).to(A.h.dtype) for _ in range(2))
    pos = torch.zeros(T, dtype=torch.int32)
    for a, b in zip(starts[:-1], starts[1:]):
        pos[a:b] = torch.arange(b - a)
    return x, d_add, torch.tensor(starts, dtype=torch.int32, device="cuda"), pos.cuda()


def call(A, x, d_add, starts, pos):
    add = A.forward(x, starts, pos)
    dx = A.backward(d_add, x, starts, pos)
    return {"add": add.clone(), "dx": dx.clone(), **{n: t.clone() for n, t in A.grad.items()}}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("starts", [[0, 30, 70], [9, 40, 41, 90], [20, 20, 128], [5, 5], [0]])
def test_rows_of_no_sequence_add_nothing(dtype, starts):
    """Behind a batch that fills all rows, and on memory that holds anything, a batch that does not is what its rows alone are."""
    tol = TOL32 if dtype == "f32" else TOL16
    used, fresh = make(128, dtype), make(128, dtype)
    call(used, *batch(used, [0, 50, 128], seed=3))
    for t in (fresh.o, fresh.dq, fresh.dk, fresh.d_qkv, fresh.q, fresh.k):
        t.fill_(float("nan"))
    x, d_add, at, pos = batch(used, starts)
    got, other = call(used, x, d_add, at, pos), call(fresh, x, d_add, at, pos)
    for n in got:
        assert torch.equal(got[n], other[n]), n
    rows = slice(starts[0], starts[-1])
    outside = torch.ones(128, dtype=torch.bool, device="cuda")
    outside[rows] = False
    for n in ("add", "dx"):
        assert (got[n][outside] == 0).all(), n
    count = starts[-1] - starts[0]
    if count == 0:
        assert all((t == 0).all() for t in got.values())
        return
    alone = make(count, dtype)
    want = call(alone, x[rows].contiguous(), d_add[rows].contiguous(), at - starts[0], pos[rows].clone())
    for n, t in want.items():
        assert far(got[n][rows] if n in ("add", "dx") else got[n], t) < tol, n


def test_scratch_of_a_graph_stays_its_own():
    """Tokens and batches that need more scratch, between the replays of a captured step of the same object; what they allocate is overwritten."""
    A, B, many = make(128, n_pos=8000), make(128, n_pos=8000), [0, 1, 2, 64, 128]
    one = batch(A, [0, 50, 128])

    def step(m):
        return m.forward(one[0], one[2], one[3]), m.backward(one[1], *(one[i] for i in (0, 2, 3)))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(A)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        add, dx = step(A)
    kept = []
    for i in range(3):
        A.start_cache(2, 2000 * (i + 1))
        A.decode(one[0][:2])
        need = S.attn_shape(2, 2, 4000 * (i + 1), A.H, A.K, A.D, A.dt, 1, 0)
        assert S.spes_attn_scratch_bytes(need, 0) > S.spes_attn_scratch_bytes(S.attn_shape(2, 128, 128, A.H, A.K, A.D, A.dt, 1, 0), 1)
        call(A, *batch(A, many, seed=6))
        kept += [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (512, 2048, 4096, 1 << 16)]
        mine = [t.clone() for t in kept]
        one[0].mul_(-0.75)
        graph.replay()
        want, want_dx = step(B)
        torch.cuda.synchronize()
        assert torch.equal(add, want) and torch.equal(dx, want_dx), i
        assert all(torch.equal(a, b) for a, b in zip(kept, mine)), i


def test_a_graph_beside_eager_calls_of_the_same_object():
    """What a replay leaves is where the optimizer step and an eager backward look for it, also behind eager calls."""
    A, B = make(128), make(128)
    first, second = batch(A, [0, 50, 128]), batch(A, [0, 100, 128], seed=4)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(A, *first)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.forward(first[0], first[2], first[3])
        A.backward(first[1], *(first[i] for i in (0, 2, 3)))
    for i in range(3):
        call(A, *second)
        first[0].mul_(-1.25)
        graph.replay()
        want = call(B, *first)
        torch.cuda.synchronize()
        for n, t in A.grad.items():
            assert torch.equal(t, want[n]), (i, n)
        assert torch.equal(A.qkv, B.qkv) and torch.equal(A.dx, want["dx"]), i
    # a graph of the backward alone, behind eager forward calls
    A.forward(first[0], first[2], first[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.backward(first[1], *(first[i] for i in (0, 2, 3)))
    for i in range(3):
        first[0].mul_(0.75)
        A.forward(first[0], first[2], first[3])
        graph.replay()
        want = call(B, *first)
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[n]) for n, t in A.grad.items()), i


def test_a_refused_token_takes_no_room():
    A = make(8)
    x = torch.randn(2, D_MODEL, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).to(A.h.dtype)
    A.start_cache(2, 1)
    with pytest.raises(S.SpesError):
        A.decode(x.float())
    assert torch.isfinite(A.decode(x)).all() and A.length.tolist() == [1, 1]


@pytest.mark.parametrize("room,n_pos", [(6, 128), (9, 6)])
@pytest.mark.parametrize("rot_dim", [None, 16, 0])
def test_replays_beyond_the_room_of_a_cache(room, n_pos, rot_dim):
    """A captured token: up to the sixth what eager calls give, then NaN, with the caches as they were; emptied caches of the same size take the graph on."""
    A, B = (make(8, n_pos=n_pos, rot_dim=rot_dim) for _ in range(2))
    x = torch.randn(6, 3, D_MODEL, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).to(A.h.dtype)
    for m in (A, B):
        m.start_cache(3, room)
        for c in m.cache:
            c.fill_(7.0)
    token = x[0].clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        A.decode(token)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = A.decode(token)
    assert A.taken == 1 and A.length.tolist() == [1, 1, 1]
    for start in (1, 0):
        if start:
            B.decode(x[0])
        else:
            for m in (A, B):
                m.start_cache(3, room)
        for i in range(start, 6):
            token.copy_(x[i])
            graph.replay()
            want = B.decode(x[i])
            torch.cuda.synchronize()
            assert torch.isfinite(out).all() and torch.equal(out, want), (start, i)
        held = [c.clone() for c in A.cache]
        for _ in range(4):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.isnan(out).all()
        assert all(torch.equal(a, b) for a, b in zip(A.cache, held)) and all((c[:, 6:] == 7.0).all() for c in A.cache)
    with pytest.raises(S.SpesError):
        B.decode(x[0])


def test_without_rotation():
    """rot_dim 0: what a rotation by no angle gives; single tokens as the whole.  (Not bit for bit: where pairs are half of the head apart a lane has chunks p and
    p + 2 of it, without rotation 2 p and 2 p + 1, so the sums over a head run in another order; within the allowance of the other tests then.)"""
    A, B = make(40, rot_dim=0), make(40)
    x, d_add, starts, pos = batch(A, [0, 30, 40])
    got, want = call(A, x, d_add, starts, pos), call(B, x, d_add, starts, torch.zeros_like(pos))
    for n in want:
        assert far(got[n], want[n]) < TOL16, n
    A.start_cache(1, 30)
    single = torch.cat([A.decode(x[i: i + 1]) for i in range(30)])
    assert far(single, got["add"][:30]) < TOL16


def test_a_backward_goes_by_the_sequences_that_it_is_given():
    """A replayed forward of three sequences behind an eager one of a single sequence, then an eager backward of the three."""
    A, B = make(128), make(128)
    three, one = batch(A, [0, 40, 90, 128]), batch(A, [0, 128], seed=8)
    A.forward(three[0], three[2], three[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.forward(three[0], three[2], three[3])
    A.forward(one[0], one[2], one[3])
    graph.replay()
    dx = A.backward(three[1], *(three[i] for i in (0, 2, 3)))
    want = call(B, *three)
    torch.cuda.synchronize()
    assert torch.equal(dx, want["dx"]) and all(torch.equal(t, want[n]) for n, t in A.grad.items())
