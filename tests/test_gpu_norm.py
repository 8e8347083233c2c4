"""Norm with residual additions: device kernels against the definition in 64 bits, element by element.

Allowances count roundings.  A row's sums are at most 64 terms one after the other and then ten levels of a tree, so every
statistic is within 80 steps of 2^-24 of its terms' magnitudes; K = 128 covers those and the handful of operations on an element.  A
result in bf16 is rounded once more, 2^-8 of it at most half a step."""
import numpy as np
import pytest
import torch

import paper_2602_11543_amd as S

pytestmark = pytest.mark.gpu

K, STEP = 128, 2.0 ** -24
LAYER, RMS = S.SPES_NORM_LAYER, S.SPES_NORM_RMS
SHAPES = [(1, 1), (1, 64), (3, 7), (5, 128), (5, 129), (17, 255), (33, 256), (2, 257), (9, 511), (9, 512), (4, 513), (7, 1001), (3, 1024),
          (6, 1025), (5, 2047), (5, 2048), (3, 2049), (2, 4096), (3, 4099), (2, 8192), (2, 8200), (1, 16384), (2, 16383), (2100, 40), (1333, 300),
          (1100, 520), (600, 1030)]


def dt(dtype):
    return S.SPES_F32 if dtype == torch.float32 else S.SPES_BF16


def half(dtype):
    return torch.finfo(dtype).eps / 2


def reference(kind, x, add, w, b, eps, dtype, dy=None, dres=None):
    """In 64 bits, with the magnitudes that the allowances are counted in."""
    r = {}
    v = x.double()
    if add is not None:
        r["sum"] = v + add.double()
        v = (x.float() + add.float()).to(dtype).double()
    n = v.shape[1]
    mean = v.mean(1, keepdim=True) if kind == LAYER else torch.zeros_like(v[:, :1])
    rstd = ((v - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    hat = (v - mean) * rstd
    w = w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    r.update(mean=mean[:, 0], rstd=rstd[:, 0], y=hat * w + b)
    # of (v - mean) rstd: the mean is off by K steps of the largest value, and so is every difference
    spread = (v.abs() + (v.abs().amax(1, keepdim=True) if kind == LAYER else 0)) * rstd
    r["y_mag"] = spread * w.abs() + b.abs() + spread * rstd * v.abs().amax(1, keepdim=True) * 0
    if dy is not None:
        dy = dy.double()
        h = dy * w
        dx = (h - hat * (h * hat).mean(1, keepdim=True) - (h.mean(1, keepdim=True) if kind == LAYER else 0)) * rstd
        mag = (h.abs() + spread * (h.abs() * spread).mean(1, keepdim=True) + (h.abs().mean(1, keepdim=True) if kind == LAYER else 0)) * rstd
        if dres is not None:
            dx, mag = dx + dres.double(), mag + dres.double().abs()
        r.update(dx=dx, dx_mag=mag, d_weight=(dy * hat).sum(0), dw_mag=(dy.abs() * spread).sum(0), d_bias=dy.sum(0), db_mag=dy.abs().sum(0))
        assert n == dx.shape[1]
    return r


def within(got, want, mag, dtype, steps, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    allow = half(dtype) * (1 + 2.0 ** -6) * want.abs() * (dtype != torch.float32) + steps * STEP * (mag + want.abs())
    worst = ((got - want).abs() - allow).max()
    assert float(worst) <= 0, (what, float(worst), float((got - want).abs().max()))


def inputs(rows, cols, dtype, kind, residual, strided, seed):
    g = torch.Generator().manual_seed(seed)
    pad = 5 if strided else 0

    def mat():
        t = torch.randn(rows, cols + pad, generator=g).to(dtype).cuda()
        return t[:, pad // 2: pad // 2 + cols]

    x = mat()
    w, b = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype).cuda(), (0.3 * torch.randn(cols, generator=g)).to(dtype).cuda()
    return dict(x=x, dy=mat(), w=w, b=b if kind == LAYER else None, add=mat() if residual else None, dres=mat() if residual else None)


def run(kind, i, eps, accumulate=None, dx_only=False):
    rows, cols = i["x"].shape
    dtype = i["x"].dtype
    new = lambda *s, t=torch.float32: torch.full(s, float("nan"), dtype=t, device="cuda")  # noqa: E731
    o = dict(y=new(rows, cols, t=dtype), rstd=new(rows), mean=new(rows) if kind == LAYER else None, sum=new(rows, cols, t=dtype) if i["add"] is not None else None)
    S.spes_norm_fwd(kind, rows, cols, dt(dtype), i["x"], i["add"], i["w"], i["b"], eps, o["sum"], o["y"], o["mean"], o["rstd"])
    o["dx"] = new(rows, cols, t=dtype)
    if not dx_only:
        o["d_weight"] = new(cols) if accumulate is None else accumulate[0].clone()
        if i["b"] is not None:
            o["d_bias"] = new(cols) if accumulate is None else accumulate[1].clone()
        scratch = torch.full((S.spes_norm_scratch_bytes(rows, cols),), 255, dtype=torch.uint8, device="cuda")
    S.spes_norm_bwd(kind, rows, cols, dt(dtype), i["dy"], i["x"] if i["add"] is None else o["sum"], i["w"], o["mean"], o["rstd"], i["dres"],
                    o["dx"], o.get("d_weight"), o.get("d_bias"), int(accumulate is not None), None if dx_only else scratch)
    torch.cuda.synchronize()
    return o


def check(kind, i, eps, o, base=None):
    rows, dtype = i["x"].shape[0], i["x"].dtype
    r = reference(kind, i["x"], i["add"], i["w"], i["b"], eps, dtype, i["dy"], i["dres"])
    if i["add"] is not None:
        within(o["sum"], r["sum"], r["sum"].abs(), dtype, 1, "sum")
    if kind == LAYER:
        within(o["mean"], r["mean"], i["x"].double().abs().amax(1) * (1 if i["add"] is None else 2), torch.float32, K, "mean")
    within(o["rstd"], r["rstd"], r["rstd"], torch.float32, K, "rstd")
    within(o["y"], r["y"], r["y_mag"], dtype, K, "y")
    within(o["dx"], r["dx"], r["dx_mag"], dtype, K, "dx")
    if "d_weight" in o:
        base = base or (torch.zeros_like(o["d_weight"]), torch.zeros_like(o["d_weight"]))
        within(o["d_weight"], r["d_weight"] + base[0].double(), r["dw_mag"] + base[0].abs(), torch.float32, K + rows / 16, "d_weight")
        if i["b"] is not None:
            within(o["d_bias"], r["d_bias"] + base[1].double(), r["db_mag"] + base[1].abs(), torch.float32, K + rows / 16, "d_bias")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", [LAYER, RMS], ids=["layer", "rms"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_backward(device, rows, cols, kind, dtype):
    for residual, strided in ((False, False), (True, False), (False, True), (True, True)):
        i = inputs(rows, cols, dtype, kind, residual, strided, rows * 31 + cols)
        check(kind, i, 1e-5, run(kind, i, 1e-5))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(33, 72), (70, 1001), (5, 3000)])
def test_added_to_the_gradients_that_are_there(device, rows, cols, dtype):
    i = inputs(rows, cols, dtype, LAYER, True, False, 3)
    base = (torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda"))
    check(LAYER, i, 1e-6, run(LAYER, i, 1e-6, accumulate=base), base)


def test_frozen_weight(device):
    i = inputs(20, 300, torch.bfloat16, LAYER, True, False, 4)
    full, only = run(LAYER, i, 1e-5), run(LAYER, i, 1e-5, dx_only=True)
    assert "d_weight" not in only and torch.equal(full["dx"], only["dx"])


@pytest.mark.parametrize("kind", [LAYER, RMS], ids=["layer", "rms"])
def test_large_offset_and_constant_rows(device, kind):
    """The mean is subtracted before anything is squared: a row of values near 1000 keeps its statistics; a constant row has variance zero."""
    i = inputs(40, 777, torch.float32, kind, False, False, 5)
    i["x"] += 1000
    i["x"][7] = 3.25
    i["x"][8] = 0
    o = run(kind, i, 1e-5)
    r = reference(kind, i["x"], None, i["w"], i["b"], 1e-5, torch.float32)
    if kind == LAYER:
        # differences of values near 1000 are exact to 2^-14; the mean is off by at most K steps of 1000 (and by that much are all of them)
        var_err = 2 * 1000 * K * STEP
        assert float(((o["rstd"].double() - r["rstd"]).abs() / r["rstd"])[[0, 1, 2, 39]].max()) < var_err
        assert float(o["mean"][7]) == 3.25 and torch.equal(o["y"][7], i["b"]) and torch.equal(o["y"][8], i["b"])
        assert abs(float(o["rstd"][7]) * 1e-5 ** 0.5 - 1) < K * STEP
    else:
        within(o["rstd"], r["rstd"], r["rstd"], torch.float32, K, "rstd")
        assert float(o["y"][8].abs().max()) == 0
    assert torch.isfinite(o["dx"]).all()


@pytest.mark.parametrize("cols", [64, 700, 5000])
def test_a_bad_row_stays_in_its_row(device, cols):
    i = inputs(37, cols, torch.bfloat16, LAYER, False, False, 6)
    want = run(LAYER, i, 1e-5)
    i["x"][5, 3], i["x"][6, 0] = float("nan"), float("inf")
    got = run(LAYER, i, 1e-5)
    keep = [r for r in range(37) if r not in (5, 6)]
    for name in ("y", "dx", "mean", "rstd"):
        assert torch.equal(got[name][keep], want[name][keep]), name
    assert torch.isnan(got["y"][5]).all() and torch.isnan(got["y"][6]).any()


def test_no_rows(device):
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    s = torch.empty(0, device="cuda")
    S.spes_norm_fwd(RMS, 0, 64, S.SPES_F32, e, None, w, None, 1e-5, None, e, None, s)
    scratch = torch.empty(S.spes_norm_scratch_bytes(0, 64), dtype=torch.uint8, device="cuda")
    dw = torch.ones(64, device="cuda")
    S.spes_norm_bwd(RMS, 0, 64, S.SPES_F32, e, e, w, None, s, None, e, dw, None, 1, scratch)
    torch.cuda.synchronize()
    assert bool((dw == 1).all())
    S.spes_norm_bwd(RMS, 0, 64, S.SPES_F32, e, e, w, None, s, None, e, dw, None, 0, scratch)
    torch.cuda.synchronize()
    assert bool((dw == 0).all())


@pytest.mark.parametrize("kind", [LAYER, RMS], ids=["layer", "rms"])
def test_gradient_against_differences(device, kind):
    """Central differences of the loss sum(dy y) in 64 bits, step 2^-17: truncation and cancellation below 2^-24 of the terms."""
    i = inputs(4, 19, torch.float32, kind, False, False, 8)
    o = run(kind, i, 1e-3)
    x, dy, step = i["x"].double(), i["dy"].double(), 2.0 ** -17
    f = lambda v, w: (reference(kind, v, None, w, i["b"], 1e-3, torch.float64)["y"] * dy).sum()  # noqa: E731
    mag = reference(kind, i["x"], None, i["w"], i["b"], 1e-3, torch.float32, i["dy"])["dx_mag"]
    for r in range(4):
        for c in range(19):
            d = torch.zeros_like(x)
            d[r, c] = step
            want = float(f(x + d, i["w"]) - f(x - d, i["w"])) / (2 * step)
            assert abs(float(o["dx"][r, c]) - want) <= 2 * K * STEP * float(mag[r].max())
    for c in range(19):
        d = torch.zeros(19, dtype=torch.float64, device="cuda")
        d[c] = step
        want = float(f(x, i["w"].double() + d) - f(x, i["w"].double() - d)) / (2 * step)
        assert abs(float(o["d_weight"][c]) - want) <= 2 * K * STEP * float(dy.abs().sum()) * 8


def test_same_bits_again_and_on_another_stream(device):
    i = inputs(3000, 520, torch.bfloat16, LAYER, True, False, 9)
    a = run(LAYER, i, 1e-5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = run(LAYER, i, 1e-5)
    torch.cuda.synchronize()
    for name in a:
        assert a[name] is None or torch.equal(a[name], b[name]), name


def test_captured_into_a_graph(device):
    """Replays between the program's own eager work give the eager bits, on changed inputs too."""
    i = inputs(300, 260, torch.bfloat16, LAYER, True, False, 10)
    rows, cols = i["x"].shape
    o = run(LAYER, i, 1e-5)
    scratch = torch.empty(S.spes_norm_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")

    def step():
        S.spes_norm_fwd(LAYER, rows, cols, S.SPES_BF16, i["x"], i["add"], i["w"], i["b"], 1e-5, o["sum"], o["y"], o["mean"], o["rstd"])
        S.spes_norm_bwd(LAYER, rows, cols, S.SPES_BF16, i["dy"], o["sum"], i["w"], o["mean"], o["rstd"], i["dres"], o["dx"], o["d_weight"], o["d_bias"], 0, scratch)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        i["x"].copy_(torch.randn(rows, cols, device="cuda").to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in o.items()}
        want = run(LAYER, i, 1e-5)
        for n in want:
            assert torch.equal(got[n], want[n]), (k, n)


def test_binding_refuses_wrong_tensors(device):
    i = inputs(8, 64, torch.float32, RMS, False, False, 11)
    y, s = torch.empty(8, 64, device="cuda"), torch.empty(8, device="cuda")
    fwd = lambda x, w=i["w"], y=y, s=s: S.spes_norm_fwd(RMS, 8, 64, S.SPES_F32, x, None, w, None, 1e-5, None, y, None, s)  # noqa: E731
    for bad in (lambda: fwd(i["x"][:7]), lambda: fwd(i["x"].t().contiguous().t()), lambda: fwd(i["x"][:1].expand(8, 64)), lambda: fwd(i["x"].cpu()),
                lambda: fwd(i["x"].bfloat16()), lambda: fwd(i["x"], w=i["w"][:63]), lambda: fwd(i["x"], s=s[:5]), lambda: fwd(i["x"], y=y.bfloat16())):
        with pytest.raises(S.SpesError):
            bad()
    g = torch.empty(64, device="cuda")
    with pytest.raises(S.SpesError):       # scratch too small
        S.spes_norm_bwd(RMS, 8, 64, S.SPES_F32, y, y, i["w"], None, s, None, i["x"], g, None, 0, torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert np.isfinite(float(i["x"].sum()))
