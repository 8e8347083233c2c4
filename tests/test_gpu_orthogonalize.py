"""Newton-Schulz orthogonalisation and the optimizer step built on it: device kernels against the formulas in 64 bits.

Allowances.  bf16 storage computes on fp16 operands, half a step of which is U = 2^-11: what the last two steps round (the others carry X with
its remainder) enters the result with weights of about 4 (X), 5 (P) and 16 (G) in the worst case and, being of random sign, with 0.41 of that added
in squares over two steps: 8 U in norm.  A bf16 result is rounded once more, 2^-8 at most and 0.41 of it in norm.  fp32 storage
takes pairs of fp16 values, 2^-22, and adds up to some thousand products in fp32: 16 of those steps.  Every 64 x 64 block is held to
four times the norm's allowance, so that an error in a corner shows."""
import numpy as np
import pytest
import torch

import paper_2602_11543_amd as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -11
ALLOW = {torch.bfloat16: 8 * U, torch.float32: 16 * 2.0 ** -22}
COEF = (3.4445, -4.7750, 2.0315)
TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


def dt(dtype):
    return S.SPES_F32 if dtype == torch.float32 else S.SPES_BF16


def exact(u, steps=5, coef=COEF):
    x = u.double().cpu()
    norm = torch.linalg.matrix_norm(x)
    x = x / norm if float(norm) != 0 else x
    a, b, c = (float(np.float32(v)) for v in coef)
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            g = x @ x.T
            x = a * x + (b * g + c * g @ g) @ x
        else:
            g = x.T @ x
            x = a * x + x @ (b * g + c * g @ g)
    return x


def matrices(n, rows, cols, seed):
    """A few strong directions above a broad floor, as weight gradients have."""
    g = torch.Generator().manual_seed(seed)
    x = 0.05 * torch.randn(n, rows, cols, generator=g)
    r = min(8, rows, cols)
    a, b = torch.randn(n, rows, r, generator=g), torch.randn(n, r, cols, generator=g)
    return x + 0.1 * (a * torch.logspace(0, -1.5, r)) @ b


def run(src, steps=5, coef=None, fill=255):
    n, rows, cols = src.shape
    out = torch.full_like(src, float("nan"))
    scratch = torch.full((S.spes_orthogonalize_scratch_bytes(n, rows, cols, dt(src.dtype)),), fill, dtype=torch.uint8, device="cuda")
    S.spes_orthogonalize(n, rows, cols, dt(src.dtype), src, out, steps, coef, scratch)
    torch.cuda.synchronize()
    return out


def near(got, want, allow, more=0.0):
    """allow: of the norm; more: absolute, of each element."""
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    d, norm = got - want, float(want.norm())
    assert float(d.norm()) <= allow * norm + more * want.numel() ** 0.5, (float(d.norm()) / max(norm, 1e-300), allow)
    rms = norm / want.numel() ** 0.5
    for r in range(0, want.shape[0], 64):
        for c in range(0, want.shape[1], 64):
            b = d[r: r + 64, c: c + 64]
            level = max(rms, float(want[r: r + 64, c: c + 64].square().mean()) ** 0.5)
            assert float(b.square().mean()) ** 0.5 <= 4 * (allow * level + more), (r, c)


def out_allow(dtype):
    return ALLOW[dtype] + (0.41 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)


@TYPES
@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (3, 1, 64), (2, 64, 1), (2, 3, 5), (1, 8, 8), (2, 64, 64), (3, 65, 63), (2, 63, 65), (1, 128, 129), (2, 130, 260),
                                         (3, 200, 100), (2, 333, 257), (4, 512, 256), (1, 1000, 72), (1, 72, 1000), (1, 515, 770), (1, 1024, 640), (25, 96, 80)])
def test_against_the_formula(device, n, rows, cols, dtype):
    src = matrices(n, rows, cols, rows + cols).to(dtype).cuda()
    out = run(src)
    for i in range(n):
        near(out[i], exact(src[i]), out_allow(dtype))


@TYPES
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
def test_other_numbers_of_steps(device, steps, dtype):
    src = matrices(2, 150, 90, 5).to(dtype).cuda()
    out = run(src, steps)
    for i in range(2):
        near(out[i], exact(src[i], steps), out_allow(dtype) * max(1, steps / 5))


@TYPES
def test_other_coefficients(device, dtype):
    """3/2 x - 1/2 x^3, which converges to singular values of 1."""
    src = matrices(1, 96, 64, 6).to(dtype).cuda()
    out = run(src, 24, (1.5, -0.5, 0.0))
    near(out[0], exact(src[0], 24, (1.5, -0.5, 0.0)), 4 * out_allow(dtype))
    gram = out[0].double().T @ out[0].double()
    assert float((gram - torch.eye(64, device="cuda")).norm()) <= 8 * (8 * out_allow(dtype))


@TYPES
def test_scale_of_the_input_does_not_matter(device, dtype):
    """The same matrix times powers of two from 2^-100 to 2^100: the same bits."""
    one = matrices(1, 70, 130, 7).to(dtype).cuda()
    src = torch.cat([one * 2.0 ** p for p in (0, -100, -40, 30, 100)])
    out = run(src)
    for i in range(1, 5):
        assert torch.equal(out[i], out[0])


@TYPES
@pytest.mark.parametrize("rows,cols", [(70, 130), (130, 70), (64, 64)])
def test_zeros_and_bad_numbers_stay_in_their_matrix(device, rows, cols, dtype):
    src = matrices(5, rows, cols, 8).to(dtype).cuda()
    want = run(src)
    src[1] = 0
    src[2, 3, 4] = float("nan")
    src[4, rows - 1, cols - 1] = float("inf")
    out = run(src)
    assert bool((out[1] == 0).all()) and torch.isnan(out[2]).all() and torch.isnan(out[4]).all()
    assert torch.equal(out[0], want[0]) and torch.equal(out[3], want[3])


@TYPES
def test_rank_one(device, dtype):
    """One singular value; the others are zero and stay near it: rounding is all there is to grow."""
    g = torch.Generator().manual_seed(9)
    src = (torch.randn(1, 90, 1, generator=g) @ torch.randn(1, 1, 150, generator=g)).to(dtype).cuda()
    if dtype == torch.float32:
        out = run(src)
        # what rounding leaves beside the one direction, 2^-22 of it in norm at most, grows 3.45-fold a step
        assert float((out[0].double().cpu() - exact(src[0])).norm()) <= 3.45 ** 5 * 4 * 2.0 ** -22
    else:
        assert torch.isfinite(run(src)).all()


@TYPES
def test_same_bits_whatever_is_in_the_scratch_and_beside_it(device, dtype):
    src = matrices(3, 200, 137, 10).to(dtype).cuda()
    a = run(src)
    assert torch.equal(a, run(src, fill=0)) and torch.equal(a[1:2], run(src[1:2].clone()))


def muon_reference(w, m, g, lr, beta, nesterov, wd, scale, grad_scale):
    g = g.double() * grad_scale
    m = beta * m.double() + g
    u = g + beta * m if nesterov else m
    return w.double() * (1 - lr * wd) - lr * scale * exact(u).to(w.device), m


def muon(device, dtype, experts, mask, rows, cols, nesterov, with_master=True, grad_scale=0.5, lr=0.02, wd=0.1, beta=0.9, seed=0, check=None):
    n = int(mask.sum())
    at = [e for e in range(experts) if mask[e]]
    g = torch.Generator().manual_seed(seed)
    p0 = (0.02 * torch.randn(experts, rows, cols, generator=g)).to(dtype).cuda()
    param, master = p0.clone(), (p0[at].float() * (1 + 2.0 ** -12) if with_master else None)
    w0 = master.clone() if with_master else p0[at].clone()
    m, grad = matrices(n, rows, cols, seed + 1).cuda(), matrices(n, rows, cols, seed + 2).cuda()
    m0 = m.clone()
    scale = 0.2 * max(rows, cols) ** 0.5
    scratch = torch.full((S.spes_orthogonalize_scratch_bytes(n, rows, cols, dt(dtype)),), 255, dtype=torch.uint8, device="cuda")
    S.spes_masked_muon(experts, rows, cols, dt(dtype), param, mask, master, m, grad, lr, beta, int(nesterov), wd, scale, 5, None, grad_scale, scratch)
    torch.cuda.synchronize()
    step = 2.0 ** -24
    f = lambda v: float(np.float32(v))  # noqa: E731
    for i in range(n) if check is None else check:
        w, mm = muon_reference(w0[i], m0[i], grad[i], f(lr), f(beta), nesterov, f(wd), f(scale), f(grad_scale))
        assert float(((m[i].double() - mm).abs() - 3 * step * (m0[i].abs() + grad[i].abs())).max()) <= 0
        got = master[i] if with_master else param[at[i]]
        delta = (w - w0[i].double() * (1 - f(lr) * f(wd))).cpu()
        near(got.cpu().double() - (w0[i].double() * (1 - f(lr) * f(wd))).cpu(), delta, ALLOW[dtype], more=4 * step * float(w0[i].abs().max()))
        if with_master:
            assert torch.equal(param[at[i]], master[i].to(dtype))
    frozen = [e for e in range(experts) if not mask[e]]
    assert torch.equal(param[frozen], p0[frozen])


@TYPES
@pytest.mark.parametrize("rows,cols", [(64, 64), (200, 328), (328, 200), (77, 35), (35, 77), (1, 16), (513, 129)])
def test_optimizer_step(device, rows, cols, dtype):
    for nesterov in (False, True):
        muon(device, dtype, 5, np.array([0, 1, 0, 1, 1], dtype=np.uint8), rows, cols, nesterov, seed=rows)


def test_f32_store_is_its_own_master(device):
    muon(device, torch.float32, 3, np.array([1, 0, 1], dtype=np.uint8), 100, 60, True, with_master=False)


@TYPES
def test_more_matrices_than_one_launch_updates(device, dtype):
    mask = np.ones(140, dtype=np.uint8)
    mask[5] = mask[70] = 0
    muon(device, dtype, 140, mask, 16, 24, True)


def test_nothing_trainable(device):
    param = torch.ones(3, 8, 8, dtype=torch.bfloat16, device="cuda")
    S.spes_masked_muon(3, 8, 8, S.SPES_BF16, param, np.zeros(3, dtype=np.uint8), None, None, None, 0.1, 0.9, 1, 0.1, 1.0)
    torch.cuda.synchronize()
    assert bool((param == 1).all())


@pytest.mark.parametrize("dtype,n,rows,cols", [(torch.bfloat16, 2, 1536, 1280), (torch.float32, 1, 768, 2048), (torch.bfloat16, 1, 2048, 2048)])
def test_larger_matrices(device, dtype, n, rows, cols):
    src = matrices(n, rows, cols, 3).to(dtype).cuda()
    out = run(src)
    near(out[0], exact(src[0]), out_allow(dtype))


# tests/test_operators_plan.py holds the sides
SIDES = [(40, 520, 780, 256), (40, 780, 520, 256), (180, 500, 761, 256), (2, 1000, 1300, 128), (4, 1000, 990, 128), (2, 300, 200, 64), (15, 250, 256, 64)]


@TYPES
@pytest.mark.parametrize("n,rows,cols,side", SIDES)
def test_every_tile(device, n, rows, cols, side, dtype):
    src = matrices(n, rows, cols, side).to(dtype).cuda()
    out = run(src)
    for i in {0, 1, n // 2, n - 1}:
        near(out[i], exact(src[i]), out_allow(dtype))
    assert torch.equal(out[n - 1:], run(src[n - 1:].clone())) or side != 64


@TYPES
@pytest.mark.parametrize("rows,cols", [(520, 780), (780, 520)])
def test_optimizer_step_on_full_tiles(device, rows, cols, dtype):
    mask = np.ones(44, dtype=np.uint8)
    mask[[0, 7, 20, 43]] = 0
    muon(device, dtype, 44, mask, rows, cols, True, check=(0, 1, 39))


@TYPES
def test_captured_into_a_graph_and_on_another_stream(device, dtype):
    src = matrices(2, 140, 300, 12).to(dtype).cuda()
    out = torch.empty_like(src)
    scratch = torch.empty(S.spes_orthogonalize_scratch_bytes(2, 140, 300, dt(dtype)), dtype=torch.uint8, device="cuda")
    step = lambda: S.spes_orthogonalize(2, 140, 300, dt(dtype), src, out, 5, None, scratch)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(out, run(src))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        src.copy_(matrices(2, 140, 300, 20 + k).to(dtype))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, run(src)), k


def test_binding_refuses_wrong_tensors(device):
    src = torch.zeros(2, 32, 48, device="cuda")
    scratch = torch.empty(S.spes_orthogonalize_scratch_bytes(2, 32, 48, S.SPES_F32), dtype=torch.uint8, device="cuda")
    for bad in (dict(src=src.half()), dict(src=src[:1]), dict(src=src.transpose(1, 2)), dict(out=src.cpu()), dict(scratch=scratch[:-1]), dict(coef=(1.0, 2.0)),
                dict(scratch=None), dict(steps=0)):
        k = dict(src=src, out=torch.empty_like(src), steps=5, coef=None, scratch=scratch)
        k.update(bad)
        with pytest.raises(S.SpesError):
            S.spes_orthogonalize(2, 32, 48, S.SPES_F32, **k)


@TYPES
@pytest.mark.parametrize("rows,cols", [(1100, 1300), (1300, 1100)])
def test_optimizer_step_on_halves_of_small_tiles(device, rows, cols, dtype):
    muon(device, dtype, 2, np.array([0, 1], dtype=np.uint8), rows, cols, True, check=(0,))
    src = matrices(1, rows, cols, 5).to(dtype).cuda()
    near(run(src)[0], exact(src[0]), out_allow(dtype))


# parts where operands are pairs, which tests/test_operators_plan.py holds; others have as many from 44 K-tiles on
PARTS = [(1, 64, 2900, 10), (4, 128, 2900, 10), (4, 2900, 128, 10), (1, 300, 4864, 8), (2, 35, 3300, 13), (1, 20, 2900, 10), (3, 100, 1500, 6)]


@TYPES
@pytest.mark.parametrize("n,rows,cols,parts", PARTS)
def test_long_contraction_in_parts(device, n, rows, cols, parts, dtype):
    src = matrices(n, rows, cols, parts).to(dtype).cuda()
    out = run(src)
    for i in {0, n - 1}:
        near(out[i], exact(src[i]), out_allow(dtype))
    assert torch.equal(out, run(src))
    muon(device, dtype, n + 1, np.array([1] * n + [0], dtype=np.uint8), rows, cols, False, check=(0,))
