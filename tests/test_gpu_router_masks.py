"""Routing where masks, biases, bad numbers and far logits meet: what counts for the choice, and gates that agree with it and with their gradient.

The choice is compared exactly with the definition in 64 bits, a masked expert left out first.  A score in 32 bits is within some 20 steps of
2^-24; sums c of a score and a bias that are nearer than 2^-18 of their size are drawn again.  Gates and gradients have K = 64 steps of their
terms, and half a step of its distance for every score that is e to the power of one."""
import itertools
import math

import pytest
import torch

import paper_2602_11543_amd as S
from test_gpu_router import K, SIGMOID, SOFTMAX, STEP, backward, forward

pytestmark = pytest.mark.gpu

INF, LOWEST = math.inf, torch.finfo(torch.float32).min
SCORES = pytest.mark.parametrize("score", [SOFTMAX, SIGMOID], ids=["softmax", "sigmoid"])


def counts(logits, bias, score):
    """c in 64 bits: s + bias, -inf where the logit is -inf, the type's lowest value or a NaN, or the sum is a NaN."""
    l = logits.double()
    s = torch.sigmoid(l) if score == SIGMOID else torch.softmax(l, 1)
    c = s if bias is None else s + bias.double()
    return torch.where((logits <= LOWEST) | c.isnan(), -INF, c)


def choose(c, groups, kept, k):
    """Indices, and whether a token's choice is clear of rounding.  Equal sums are clear where they are -inf."""
    T, M = c.shape
    size = 1 + c.abs().masked_fill(c.isinf(), 0).amax(1, keepdim=True)
    clear = torch.ones(T, dtype=torch.bool, device=c.device)

    def apart(v):
        return ((v[:, :-1] - v[:, 1:] > 2.0 ** -18 * size) | (v[:, 1:] == -INF)).all(1)

    if groups > 1:
        two = c.view(T, groups, M // groups).sort(2, descending=True).values[:, :, :2]
        best = torch.where(two == -INF, 0.0, two).sum(2).masked_fill(two[:, :, 0] == -INF, -INF).sort(dim=1, descending=True, stable=True)
        if kept < groups:
            clear &= apart(best.values[:, kept - 1: kept + 1])
        open_ = torch.zeros(T, groups, dtype=torch.bool, device=c.device).scatter_(1, best.indices[:, :kept], True)
        inside = open_.repeat_interleave(M // groups, 1)
    else:
        inside = torch.ones_like(c, dtype=torch.bool)
    # in open groups first, then by c, then by number
    order = c.sort(dim=1, descending=True, stable=True)
    first = inside.gather(1, order.indices).to(torch.int8).sort(dim=1, descending=True, stable=True).indices
    idx, v = order.indices.gather(1, first), order.values.gather(1, first)
    n = min(k + 1, kept * (M // groups))
    return idx[:, :k], clear & apart(v[:, :n])


@SCORES
@pytest.mark.parametrize("groups,kept,k", [(1, 1, 6), (6, 2, 6), (6, 6, 16), (16, 3, 4), (3, 1, 2)])
@pytest.mark.parametrize("low", [-INF, LOWEST], ids=["inf", "lowest"])
def test_masked_experts_with_a_bias(device, score, groups, kept, k, low):
    """An expert that a token must not get is not chosen for its bias, and does not open its group."""
    T, M = 200, 48
    g = torch.Generator().manual_seed(groups)
    bias = (0.5 * torch.randn(M, generator=g)).cuda()
    hide = torch.rand(T, M, generator=g) < torch.rand(T, 1, generator=g)          # from a few experts to nearly all
    hide[3] = True
    for b in (bias, None):
        logits = torch.randn(T, M, generator=g)
        for _ in range(60):
            dev = logits.masked_fill(hide, low).cuda()
            bad = ~choose(counts(dev, b, score), groups, kept, k)[1].cpu()
            if not bool(bad.any()):
                break
            logits[bad] = torch.randn(int(bad.sum()), M, generator=g)
        assert not bool(bad.any())
        want = choose(counts(dev, b, score), groups, kept, k)[0]
        for renorm in (0, 1):
            idx, gate, count = forward(dev, b, k, S.router_opts(score, groups, kept, renorm, 1.0))
            assert torch.equal(idx.long(), want)
            assert torch.equal(count.long(), torch.bincount(want.reshape(-1), minlength=M))
            masked = hide.cuda().gather(1, want)
            masked[hide.all(1)] = False
            assert bool((gate[masked] == 0).all()) and bool(torch.isfinite(gate).all())


def test_underflowing_scores_without_a_bias(device):
    """An expert whose probability is too small for 32 bits is still ahead of a masked one of a lower number."""
    logits = torch.full((5, 40), -INF, device="cuda")
    logits[:, 30], logits[:, 20], logits[:, 25] = 400.0, 0.0, -300.0
    idx, gate, _ = forward(logits, None, 3, S.router_opts(SOFTMAX))
    assert torch.equal(idx.long(), torch.tensor([30, 20, 25], device="cuda").expand(5, 3))
    assert torch.equal(gate, torch.tensor([1.0, 0.0, 0.0], device="cuda").expand(5, 3))


def test_a_group_of_bad_numbers_does_not_open(device):
    """A NaN is passed over wherever it stands in its group: it does not stand in for a second score."""
    M, groups = 24, 3
    for at in range(8):
        for other in range(8):
            if other == at:
                continue
            logits = torch.full((1, M), -2.0, device="cuda")
            logits[0, at], logits[0, other] = math.nan, 3.0                 # 0.95 + 0.12
            logits[0, 8:16] = -4.0
            logits[0, 10], logits[0, 13] = 0.5, 0.4                         # 0.62 + 0.60, which wins
            idx, gate, _ = forward(logits, None, 3, S.router_opts(SIGMOID, groups, 1))
            assert idx.tolist() == [[10, 13, 8]], (at, other)
            assert bool(torch.isfinite(gate).all())


@SCORES
def test_the_choice_agrees_with_the_gates(device, score):
    """Logits a few steps of 2^-24 apart: gates without renormalisation, which are the scores, descend, equal ones by expert; none is left out for
    a smaller one."""
    T, M = 4000, 16
    g = torch.Generator().manual_seed(5)
    base = 2 * torch.randn(T, 1, generator=g)
    logits = (base * (1 + 2.0 ** -23 * torch.randint(-6, 7, (T, M), generator=g))).cuda()
    idx, gate, _ = forward(logits, None, 16, S.router_opts(score))
    ahead, behind = gate[:, :-1], gate[:, 1:]
    assert bool(((ahead > behind) | ((ahead == behind) & (idx[:, :-1] < idx[:, 1:]))).all())
    few, fgate, _ = forward(logits, None, 5, S.router_opts(score))
    assert torch.equal(few, idx[:, :5]) and torch.equal(fgate, gate[:, :5])


@SCORES
@pytest.mark.parametrize("depth", [-60.0, -88.0, -95.0, -120.0, -150.0])
def test_shares_far_below_the_largest_logit(device, score, depth):
    """A bias takes experts whose logits are far down: their shares are as if nothing were above them, and so is the gradient."""
    T, M, k = 64, 32, 4
    g = torch.Generator().manual_seed(int(-depth))
    logits = torch.randn(T, M, generator=g)
    if score == SIGMOID:
        logits += depth
    else:
        logits[:, 8:] += depth
    logits = logits.cuda()
    bias = torch.zeros(M, device="cuda")
    for place, e in enumerate((9, 15, 20, 31)):
        bias[e] = 3.0 - 0.25 * place
    o = S.router_opts(score, 1, 1, 1, 2.5)
    idx, gate, _ = forward(logits, bias, k, o)
    assert torch.equal(idx.long(), torch.tensor([9, 15, 20, 31], device="cuda").expand(T, k))
    x = logits.double().gather(1, idx.long()).requires_grad_(True)
    share = torch.softmax(x, 1) if score == SOFTMAX else torch.sigmoid(x) / torch.sigmoid(x).sum(1, keepdim=True)
    allow = (K + 1 + x.detach().abs().amax()) * STEP
    assert bool(((gate - 2.5 * share).abs() <= allow * 2.5 * share).all())
    dgate = torch.randn(T, k, generator=g).cuda()
    d = backward(logits, idx, dgate, o)
    want, = torch.autograd.grad((2.5 * share * dgate.double()).sum(), x)
    size = 2.5 * share.detach() * (dgate.abs().amax(1, keepdim=True) * 2)
    assert bool(((d.gather(1, idx.long()) - want).abs() <= 2 * allow * size).all())
    rest = torch.ones_like(d, dtype=torch.bool).scatter(1, idx.long(), False)
    assert bool((d[rest] == 0).all())


@SCORES
def test_gates_of_zero_have_no_gradient(device, score):
    """Where nothing is left of the scores, forward and backward say so alike."""
    M, k = 32, 4
    logits = torch.randn(6, M, generator=torch.Generator().manual_seed(1)).cuda()
    logits[0] = -INF
    if score == SIGMOID:
        logits[1] -= 300
        logits[2] = LOWEST
    else:
        logits[1, 8:] = -INF
    bias = torch.zeros(M, device="cuda")
    bias[10:14] = 2.0
    for renorm, b in itertools.product((0, 1), (bias, None)):
        o = S.router_opts(score, 1, 1, renorm, 1.0)
        idx, gate, _ = forward(logits, b, k, o)
        d = backward(logits, idx, torch.arange(1.0, 7 * k - k + 1, device="cuda").view(6, k), o)
        none = (gate == 0).all(1)
        assert bool(none[0]) and torch.isfinite(gate).all() and torch.isfinite(d).all()
        assert bool((d[none] == 0).all())
        if score == SIGMOID:
            assert bool(none[1]) and bool(none[2])
        assert not bool(none[3:].any())
        assert bool(((gate != 0) | (d.gather(1, idx.long()) == 0)).all())


def test_a_bad_logit_shows_in_the_gates(device):
    """One NaN or +inf among a token's logits: every softmax score is NaN, and so are the gates, whichever experts stand there."""
    logits = torch.randn(4, 64, device="cuda")
    logits[1, 40], logits[2, 50] = math.nan, INF
    for renorm in (0, 1):
        _, gate, _ = forward(logits, None, 4, S.router_opts(SOFTMAX, 1, 1, renorm, 1.0))
        assert torch.isnan(gate[1:3]).all() and torch.isfinite(gate[[0, 3]]).all()
