"""The expert layer behind a routing that the caller made, and the block that runs norm, routing, experts and optimizer together."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2602_11543_amd as S
from harness import TOL, DeviceLayer, rel_err
from paper_2602_11543_amd.block import DeviceBlock
from spes_workloads import CONFIGS, layer_inputs

pytestmark = pytest.mark.gpu


def routed(L, idx, gate):
    n = len(L.trainable)
    o = dict(y=torch.full_like(L.y, float("nan")), count=torch.empty_like(L.count), dx=torch.full_like(L.dx, float("nan")),
             dgate=torch.full_like(L.gate, float("nan")), ctx=torch.full_like(L.ctx, 255))
    o["w"] = [torch.full_like(w, float("nan")) for w in (L.d_w_gate, L.d_w_up, L.d_w_down)] if n else [None] * 3
    S.spes_moe_fwd_routed(L.shape, L.x, idx, gate, L.w_gate, L.w_up, L.w_down, o["y"], o["count"], o["ctx"])
    S.spes_moe_bwd_routed(L.shape, L.dy, L.x, L.w_gate, L.w_up, L.w_down, o["ctx"], L.mask, o["dx"], o["dgate"], *o["w"])
    torch.cuda.synchronize()
    return o


@pytest.mark.parametrize("name", ["cfg1", "cfg2_small"])
def test_with_the_layers_own_choice(device, name):
    """The same choice and gates: the experts' results in the same bits; dx without the router's part."""
    L = DeviceLayer(layer_inputs(CONFIGS[name]), device)
    L.fwd(); L.bwd(); torch.cuda.synchronize()
    o = routed(L, L.idx.clone(), L.gate.clone())
    assert torch.equal(o["y"], L.y) and torch.equal(o["count"], L.count)
    assert torch.equal(o["dgate"], L.view("dgate"))
    for got, want in zip(o["w"], (L.d_w_gate, L.d_w_up, L.d_w_down)):
        assert torch.equal(got, want)
    want = L.dx.double() - L.view("dlogits").double() @ L.w_router.double()
    assert rel_err(o["dx"].double().cpu().numpy(), want.cpu().numpy()) < 2 * TOL[L.cfg.dtype]


def test_entries_that_are_no_expert(device):
    L = DeviceLayer(layer_inputs(CONFIGS["cfg1"]), device)
    L.fwd(); torch.cuda.synchronize()
    idx, gate = L.idx.clone(), L.gate.clone()
    idx[3, 0], gate[3, 0] = 0, 0.0
    idx[9, 1], gate[9, 1] = 0, 0.0
    want = routed(L, idx, gate)
    idx[3, 0], gate[3, 0] = -1, 7.0
    idx[9, 1], gate[9, 1] = 1 << 30, float("nan")
    got = routed(L, idx, gate)
    for name in ("y", "count", "dx", "dgate"):
        assert torch.equal(got[name], want[name]), name


def test_block_gradients(device):
    """A small block in fp32 against automatic differentiation of the same block in 64 bits, the choice held fixed; each of the three
    operators in a row is within the layer's tolerance."""
    T, d, M, f, k = 40, 64, 8, 32, 3
    B = DeviceBlock(T, d, M, f, k, np.array([1, 0, 1, 1, 0, 0, 1, 0]), "f32", groups=4, kept_groups=3, scale=1.5, seed=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, add, d_out = (torch.randn(T, d, device="cuda", generator=g) for _ in range(3))
    B.bias.copy_(0.05 * torch.randn(M, device="cuda", generator=g))
    B.norm_w.copy_(1 + 0.2 * torch.randn(d, device="cuda", generator=g))
    out = B.forward(x, add).clone()
    dx = B.backward(d_out)
    torch.cuda.synchronize()
    leaf = lambda t: t.double().cpu().requires_grad_(True)  # noqa: E731
    xs, nw, wr = leaf(x + add), leaf(B.norm_w), leaf(B.w_router)
    wg, wu, wd = (leaf(w) for w in B.experts.values())
    h = xs * (xs.square().mean(1, keepdim=True) + 1e-6) ** -0.5 * nw
    s = torch.sigmoid(h @ wr.t())
    idx = B.idx.long().cpu()
    sj = s.gather(1, idx)
    gate = 1.5 * sj / sj.sum(1, keepdim=True)
    a, b = torch.einsum("td,efd->tef", h, wg), torch.einsum("td,efd->tef", h, wu)
    ye = torch.einsum("tef,edf->ted", torch.nn.functional.silu(a) * b, wd)
    want = xs + (gate[:, :, None] * ye.gather(1, idx[:, :, None].expand(T, k, d))).sum(1)
    want.backward(d_out.double().cpu())
    n = lambda t: t.detach().double().cpu().numpy()  # noqa: E731
    tol = 3 * TOL["f32"]
    assert rel_err(n(out), n(want)) < tol
    assert rel_err(n(dx), n(xs.grad)) < tol
    assert rel_err(n(B.d_norm_w), n(nw.grad)) < tol
    assert rel_err(n(B.d_w_router), n(wr.grad)) < tol
    for got, w in zip(B.grad.values(), (wg, wu, wd)):
        assert rel_err(n(got), n(w.grad)[[0, 2, 3, 6]]) < tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_lowers_the_loss(device, dtype):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import block_step
    losses, loads = block_step.train(tokens=512, d_model=128, n_experts=16, d_ff=96, top_k=2, groups=4, kept_groups=2, trainable=8, steps=12, dtype=dtype,
                                     report=lambda *_: None)
    assert all(np.isfinite(losses)) and losses[-1] < 0.9 * losses[0], losses
