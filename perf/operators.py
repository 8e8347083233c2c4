"""The operators around the expert layer as a training program calls them, as a list of cases that can be timed and compared.

    norm     layer norm or root-mean-square norm in front of a block, with the residual stream's addition on the way in and the residual
             gradient's on the way back: `forward` alone, or a `step` of forward and backward with the weight's and the bias's gradients
    router   scores to experts: softmax or sigmoid, a bias that only steers the choice, groups of experts, top-k, renormalised and
             scaled weights, the load of each expert: `forward`, or a `step` with the scores' gradient
    ortho    Newton-Schulz orthogonalisation of a stack of matrices
    muon     the optimizer step built on it: momentum, orthogonalised update, weight decay, for the trainable experts of a store

Each case is one pass through the public entry points (`own`), or the same in elementary operations in 32 bits.  Shapes are the
repository's own layer workloads and sizes around them.
"""
import math

import numpy as np
import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)
STEPS = 5
LAYER, RMS = 0, 1
SOFTMAX, SIGMOID = 0, 1


def _norm(name, mode, kind, rows, cols, dtype, residual, strided):
    return dict(name=name, op="norm", mode=mode, kind=kind, rows=rows, cols=cols, dtype=dtype, residual=residual, strided=strided)


def _router(name, mode, T, M, k, score, bias, groups, kept, renorm, scale):
    return dict(name=name, op="router", mode=mode, T=T, M=M, k=k, score=score, bias=bias, groups=groups, kept=kept, renorm=renorm, scale=scale)


def _ortho(name, n, rows, cols, dtype):
    return dict(name=name, op="ortho", n=n, rows=rows, cols=cols, dtype=dtype)


def _muon(name, experts, trainable, rows, cols, dtype, nesterov=True, lr=1e-4):
    return dict(name=name, op="muon", experts=experts, trainable=trainable, rows=rows, cols=cols, dtype=dtype, nesterov=nesterov, lr=lr)


def listed():
    return [
        # scoring one short sequence: the norm ahead of the layer, where a launch's latency is what counts
        _norm("norm_short", "forward", LAYER, 200, 2048, "bf16", False, False),
        # a micro-batch of 2 x 2048 tokens of the smallest training workload
        _norm("norm_paper_1b", "step", RMS, 4096, 768, "bf16", True, False),
        # full precision, an odd width and rows that are cut out of wider ones
        _norm("norm_ragged_f32", "step", LAYER, 1531, 1001, "f32", False, True),
        # the widest training workload, with both residual additions
        _norm("norm_cfg3", "step", LAYER, 32768, 4096, "bf16", True, False),
        # a serving step: a few dozen single tokens
        _router("router_decode", "forward", 48, 64, 8, SOFTMAX, False, 1, 1, True, 1.0),
        # many small experts in groups, balanced by the bias: the form that keeps a token's experts on few devices
        _router("router_groups", "step", 16384, 256, 8, SIGMOID, True, 8, 4, True, 2.5),
        # a last batch that is not full, an expert count that is no power of two
        _router("router_ragged", "step", 3777, 160, 6, SOFTMAX, True, 5, 3, False, 1.0),
        # the widest training workload's tokens and experts
        _router("router_cfg3", "step", 32768, 64, 8, SIGMOID, True, 1, 1, True, 1.0),
        # the full-precision workload's gate matrices
        _ortho("ortho_cfg1_f32", 4, 512, 256, "f32"),
        # the one expert that a node of the 2B-shaped model trains, its down projection: more rows than columns
        _muon("muon_paper_2b", 16, 1, 1536, 1280, "bf16"),
        # one matrix of the 16 trainable experts of 64
        _muon("muon_cfg2", 64, 16, 1024, 2048, "bf16"),
        # the largest experts
        _muon("muon_cfg4", 32, 8, 4864, 3584, "bf16", nesterov=False),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)


def draw(rng):
    """Another case of the same ranges: 1 to 32768 rows of 64 to 8192 columns, 1 to 32768 tokens over 4 to 512 experts, matrices with sides
    of 64 to 4864."""
    op = rng.choice(["norm", "norm", "router", "router", "ortho", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        while True:
            rows, cols = _log(rng, 1, 32768), _log(rng, 64, 8192, rng.choice([1, 8, 64]))
            if rows * cols * (2 if dtype == "f32" else 1) <= 32768 * 4096:
                break
        return dict(op=op, mode=rng.choice(["forward", "step", "step"]), kind=rng.choice([LAYER, RMS]), rows=rows, cols=cols, dtype=dtype,
                    residual=rng.random() < 0.5, strided=rng.random() < 0.3)
    if op == "router":
        groups = rng.choice([1, 1, 2, 4, 8, rng.randint(2, 16)])
        size = rng.randint(max(1, 4 // groups), max(1, 512 // groups)) if groups > 1 else rng.choice([8, 16, 32, 64, 128, 256, rng.randint(4, 512)])
        kept = rng.randint(1, groups)
        k = rng.randint(1, min(16, kept * size))
        # (one renormalised gate is a constant, its gradient nothing)
        return dict(op=op, mode=rng.choice(["forward", "step", "step"]), T=_log(rng, 1, 32768), M=groups * size, k=k, score=rng.choice([SOFTMAX, SIGMOID]),
                    bias=rng.random() < 0.6, groups=groups, kept=kept, renorm=k > 1 and rng.random() < 0.6, scale=rng.choice([1.0, 2.5]))
    while True:
        rows, cols = _log(rng, 64, 4864, rng.choice([1, 8, 64]) if op == "ortho" else 8), _log(rng, 64, 4864, rng.choice([1, 8, 64]) if op == "ortho" else 8)
        n = rng.choice([1, 2, 4, 8, 16, rng.randint(1, 24)])
        lo, hi = min(rows, cols), max(rows, cols)
        if n * lo * lo * (3 * hi + lo) <= (0.3 if dtype == "f32" else 1.0) * 8 * 3584 * 3584 * (3 * 4864 + 3584) and n * rows * cols <= 8 * 3584 * 4864:
            break
    if op == "ortho":
        return dict(op=op, n=n, rows=rows, cols=cols, dtype=dtype)
    return dict(op=op, experts=n + rng.randint(0, 2 * n), trainable=n, rows=rows, cols=cols, dtype=dtype, nesterov=rng.random() < 0.5,
                lr=rng.choice([5e-5, 1e-4]))


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _mask(experts, trainable):
    """Which experts of the store train: spread over it, as the node's share of them is."""
    mask = np.zeros(experts, dtype=np.uint8)
    for i in range(trainable):
        mask[i * experts // trainable] = 1
    return mask


def _gradients(n, rows, cols, g):
    """Matrices with the spectrum of a weight gradient: a few strong directions above a broad floor."""
    x = 0.05 * torch.randn(n, rows, cols, device="cuda", generator=g)
    r = min(16, rows, cols)
    a, b = torch.randn(n, rows, r, device="cuda", generator=g), torch.randn(n, r, cols, device="cuda", generator=g)
    a *= torch.logspace(0, -1.5, r, device="cuda")
    for i in range(n):
        x[i].addmm_(a[i], b[i], alpha=0.1)
    return x.mul_(1e-2)


def _ambiguous(case, logits, bias):
    """Tokens whose choice of experts could hinge on the rounding of a score in 32 bits."""
    s = (torch.softmax if case["score"] == SOFTMAX else lambda l, _: torch.sigmoid(l))(logits.double(), 1)
    b = torch.zeros(case["M"], device="cuda", dtype=torch.float64) if bias is None else bias.double()
    c, size = s + b, s + b.abs()
    bad = torch.zeros(logits.shape[0], dtype=torch.bool, device="cuda")
    if case["groups"] > 1:
        per = c.view(-1, case["groups"], case["M"] // case["groups"])
        score = per.topk(min(2, per.shape[2]), 2).values.sum(2)
        v = score.sort(1, descending=True)
        if case["kept"] < case["groups"]:
            a, z = v.values[:, case["kept"] - 1], v.values[:, case["kept"]]
            bad |= a - z < 8e-6 * size.amax(1)
        chosen = torch.zeros_like(score, dtype=torch.bool).scatter_(1, v.indices[:, : case["kept"]], True)
        c = torch.where(chosen[:, :, None].expand_as(per).reshape(c.shape), c, torch.full_like(c, -1e9))
    v = c.topk(min(case["k"] + 1, case["kept"] * (case["M"] // case["groups"])), 1)
    near = size.gather(1, v.indices)
    return bad | (v.values[:, :-1] - v.values[:, 1:] < 4e-6 * torch.maximum(near[:, :-1], near[:, 1:])).any(1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *size: torch.randn(*size, device="cuda", generator=g)  # noqa: E731
    st = {"case": case}
    if case["op"] == "norm":
        rows, cols, t = case["rows"], case["cols"], _type(case)
        wide = cols + 24 if case["strided"] else cols
        # activations: features of unequal size, tokens of unequal offset
        size = 0.5 + torch.rand(wide, device="cuda", generator=g)
        x = (normal(rows, wide) * size + 0.5 * normal(rows, 1)).to(t)
        st["x"] = x[:, :cols]
        st["dy"] = normal(rows, cols).to(t)
        st["weight"] = (1 + 0.1 * normal(cols)).to(t)
        st["bias"] = (0.1 * normal(cols)).to(t) if case["kind"] == LAYER else None
        st["add"] = normal(rows, cols).to(t) if case["residual"] else None
        st["dres"] = normal(rows, cols).to(t) if case["residual"] and case["mode"] == "step" else None
    elif case["op"] == "router":
        T, M = case["T"], case["M"]
        skew = 0.5 * normal(M)
        st["bias"] = 0.1 * normal(M) * (1.0 if case["score"] == SIGMOID else 1.0 / M) if case["bias"] else None
        logits = normal(T, M) + skew
        for _ in range(40):
            bad = _ambiguous(case, logits, st["bias"])
            if not bool(bad.any()):
                break
            logits[bad] = normal(int(bad.sum()), M) + skew
        st["logits"] = logits
        st["dgate"] = normal(T, case["k"])
    elif case["op"] == "ortho":
        st["src"] = _gradients(case["n"], case["rows"], case["cols"], g).to(_type(case))
    else:
        rows, cols, mask = case["rows"], case["cols"], _mask(case["experts"], case["trainable"])
        st["mask"] = mask
        st["at"] = torch.tensor([e for e in range(case["experts"]) if mask[e]], device="cuda")
        st["param"] = (0.02 * normal(case["experts"], rows, cols)).to(_type(case))
        # trained for a while: the 32-bit weights have bits that the stored ones lack
        st["master"] = st["param"][st["at"]].float()
        if case["dtype"] == "bf16":
            st["master"] *= 1 + 2.0 ** -10 * (torch.rand(case["trainable"], rows, cols, device="cuda", generator=g) - 0.5)
        st["m"] = _gradients(case["trainable"], rows, cols, g)
        st["grad"] = _gradients(case["trainable"], rows, cols, g)
        st["scale"] = 0.2 * math.sqrt(max(rows, cols))
    return st


# ---- the plain forms ----

BETA, DECAY, EPS = 0.95, 0.1, 1e-5


def _plain_norm(case, st):
    t, out = _type(case), {}
    x = st["x"]
    if case["residual"]:
        x = (x.float() + st["add"].float()).to(t)
        out["sum"] = x
    x = x.float()
    if case["kind"] == LAYER:
        out["mean"] = mean = x.mean(1)
        x = x - mean[:, None]
    out["rstd"] = rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    hat = x * rstd[:, None]
    w = st["weight"].float()
    y = hat * w
    if st["bias"] is not None:
        y = y + st["bias"].float()
    out["y"] = y.to(t)
    if case["mode"] == "forward":
        return out
    dy = st["dy"].float()
    out["d_weight"] = (dy * hat).sum(0)
    if st["bias"] is not None:
        out["d_bias"] = dy.sum(0)
    h = dy * w
    dx = h - hat * (h * hat).mean(1, keepdim=True)
    if case["kind"] == LAYER:
        dx = dx - h.mean(1, keepdim=True)
    dx = dx * rstd[:, None]
    if st["dres"] is not None:
        dx = dx + st["dres"].float()
    out["dx"] = dx.to(t)
    return out


def _plain_scores(case, logits):
    if case["score"] == SIGMOID:
        return 1.0 / (1.0 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_router(case, st):
    T, M, k = case["T"], case["M"], case["k"]
    s = _plain_scores(case, st["logits"])
    c = s if st["bias"] is None else s + st["bias"]
    if case["groups"] > 1:
        per = c.view(T, case["groups"], M // case["groups"])
        best = per.sort(2, descending=True).values[:, :, : min(2, per.shape[2])].sum(2)
        order = best.sort(dim=1, descending=True, stable=True).indices[:, : case["kept"]]
        inside = torch.zeros_like(best, dtype=torch.bool).scatter(1, order, True)
        c = torch.where(inside[:, :, None], per, -math.inf).reshape(T, M)
    idx = c.sort(dim=1, descending=True, stable=True).indices[:, :k]
    chosen = s.gather(1, idx)
    total = chosen.sum(1, keepdim=True) if case["renorm"] else torch.ones_like(chosen[:, :1])
    gate = chosen / total * case["scale"]
    count = torch.zeros(M, dtype=torch.int32, device="cuda").scatter_add(0, idx.reshape(-1), torch.ones(T * k, dtype=torch.int32, device="cuda"))
    out = {"idx": idx.to(torch.int32), "gate": gate, "count": count}
    if case["mode"] == "forward":
        return out
    dg = st["dgate"] * case["scale"]
    if case["renorm"]:
        dg = (dg - (dg * chosen / total).sum(1, keepdim=True)) / total
    ds = torch.zeros_like(s).scatter(1, idx, dg)
    out["dlogits"] = ds * s * (1.0 - s) if case["score"] == SIGMOID else s * (ds - (ds * s).sum(1, keepdim=True))
    return out


def _plain_ortho(u):
    """u [n, rows, cols] in 32 bits; the products are with the smaller Gram matrix."""
    x = u / torch.sqrt((u * u).sum((1, 2), keepdim=True))
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    a, b, c = COEF
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2) if tall else x


def _plain_muon(case, st):
    m = st["m"].mul_(BETA).add_(st["grad"])
    u = st["grad"] + BETA * m if case["nesterov"] else m
    w = st["master"].mul_(1.0 - case["lr"] * DECAY).add_(_plain_ortho(u), alpha=-case["lr"] * st["scale"])
    st["param"][st["at"]] = w.to(st["param"].dtype)
    return {"param": st["param"], "master": w, "m": m}


# ---- the framework's calls ----


def _kept(st, name, make):
    """A buffer that the program makes once and keeps."""
    if name not in st:
        st[name] = make()
    return st[name]


def _own(st):
    import paper_2602_11543_amd as S

    case = st["case"]
    op = case["op"]
    dt = S.SPES_F32 if case.get("dtype", "f32") == "f32" else S.SPES_BF16
    if op == "norm":
        rows, cols, step = case["rows"], case["cols"], case["mode"] == "step"

        def make():
            f = lambda *size: torch.empty(*size, device="cuda", dtype=torch.float32)  # noqa: E731
            row = lambda: torch.empty(rows, cols, device="cuda", dtype=_type(case))  # noqa: E731
            o = {"rstd": f(rows), "y": row()}
            if case["kind"] == LAYER:
                o["mean"] = f(rows)
            if case["residual"]:
                o["sum"] = row()
            if step:
                o["dx"], o["d_weight"] = row(), f(cols)
                if st["bias"] is not None:
                    o["d_bias"] = f(cols)
            return o, torch.empty(S.spes_norm_scratch_bytes(rows, cols), device="cuda", dtype=torch.uint8) if step else None

        o, scratch = _kept(st, "out", make)
        S.spes_norm_fwd(case["kind"], rows, cols, dt, st["x"], st["add"], st["weight"], st["bias"], EPS, o.get("sum"), o["y"], o.get("mean"), o["rstd"])
        if step:
            S.spes_norm_bwd(case["kind"], rows, cols, dt, st["dy"], o.get("sum", st["x"]), st["weight"], o.get("mean"), o["rstd"], st["dres"], o["dx"],
                            o["d_weight"], o.get("d_bias"), 0, scratch)
        return o
    if op == "router":
        T, M, k, step = case["T"], case["M"], case["k"], case["mode"] == "step"

        def make():
            o = {"idx": torch.empty(T, k, device="cuda", dtype=torch.int32), "gate": torch.empty(T, k, device="cuda"),
                 "count": torch.empty(M, device="cuda", dtype=torch.int32)}
            if step:
                o["dlogits"] = torch.empty(T, M, device="cuda")
            return o, S.router_opts(case["score"], case["groups"], case["kept"], int(case["renorm"]), case["scale"])

        o, opts = _kept(st, "out", make)
        S.spes_router_fwd(T, M, k, opts, st["logits"], st["bias"], o["idx"], o["gate"], o["count"])
        if step:
            S.spes_router_bwd(T, M, k, opts, st["logits"], o["idx"], st["dgate"], o["dlogits"])
        return o
    n = case["n"] if op == "ortho" else case["trainable"]
    rows, cols = case["rows"], case["cols"]
    scratch = _kept(st, "scratch", lambda: torch.empty(S.spes_orthogonalize_scratch_bytes(n, rows, cols, dt), device="cuda", dtype=torch.uint8))
    if op == "ortho":
        out = _kept(st, "out", lambda: torch.empty_like(st["src"]))
        S.spes_orthogonalize(n, rows, cols, dt, st["src"], out, STEPS, None, scratch)
        return {"out": out}
    S.spes_masked_muon(case["experts"], rows, cols, dt, st["param"], st["mask"], st["master"], st["m"], st["grad"], case["lr"], BETA,
                       int(case["nesterov"]), DECAY, st["scale"], STEPS, None, 1.0, scratch)
    return {"param": st["param"], "master": st["master"], "m": st["m"]}


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "norm":
        return _plain_norm(case, state)
    if case["op"] == "router":
        return _plain_router(case, state)
    if case["op"] == "ortho":
        return {"out": _plain_ortho(state["src"].float()).to(_type(case))}
    return _plain_muon(case, state)


def work(case):
    """Every input once, every output once; a symmetric product counts half, as half of it gives the other."""
    es = 4 if case.get("dtype", "f32") == "f32" else 2
    if case["op"] == "norm":
        n, step = case["rows"] * case["cols"], case["mode"] == "step"
        passes = 2 + (2 if case["residual"] else 0) + ((3 + (1 if case["residual"] else 0)) if step else 0)
        return {"bytes": passes * n * es + 8 * case["rows"] * (2 if step else 1) + case["cols"] * 2 * (es + 4), "flops": n * (18 if step else 8)}
    if case["op"] == "router":
        T, M, k, step = case["T"], case["M"], case["k"], case["mode"] == "step"
        return {"bytes": T * M * 4 * (3 if step else 1) + T * k * (16 if step else 8) + 8 * M, "flops": T * M * (12 if step else 6)}
    lo, hi = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    n = case["n"] if case["op"] == "ortho" else case["trainable"]
    # orthogonalisation: the matrices in and out; the step: gradient, momentum and weights in, momentum, weights and their stored copy out
    moved = 2 * es if case["op"] == "ortho" else 20 + (2 if es == 2 else 0)
    return {"bytes": n * lo * hi * moved, "flops": n * STEPS * lo * lo * (3.0 * hi + lo)}


# ---- the definitions in 64 bits ----


def _exact_norm(case, st):
    out, x = {}, st["x"].double()
    if case["residual"]:
        out["sum"] = x + st["add"].double()
        x = out["sum"].to(_type(case)).double()          # the sum is normalised as it is stored
    x.requires_grad_(True)
    w = st["weight"].double().requires_grad_(True)
    b = None if st["bias"] is None else st["bias"].double().requires_grad_(True)
    mean = x.mean(1, keepdim=True) if case["kind"] == LAYER else 0.0
    var = (x - mean).square().mean(1, keepdim=True)
    y = (x - mean) / (var + EPS).sqrt() * w
    y = y if b is None else y + b
    if case["mode"] == "step":
        grads = torch.autograd.grad(y, [x, w] + ([] if b is None else [b]), st["dy"].double())
        out["dx"] = grads[0] if st["dres"] is None else grads[0] + st["dres"].double()
        out["d_weight"] = grads[1]
        if b is not None:
            out["d_bias"] = grads[2]
    if case["kind"] == LAYER:
        out["mean"] = mean.detach()[:, 0]
    out["rstd"] = (var.detach()[:, 0] + EPS) ** -0.5
    out["y"] = y.detach()
    return out


def _exact_router(case, st):
    logits = st["logits"].double().requires_grad_(True)
    s = torch.sigmoid(logits) if case["score"] == SIGMOID else torch.softmax(logits, 1)
    c = s.detach() + (0.0 if st["bias"] is None else st["bias"].double())
    size = case["M"] // case["groups"]
    best = c.view(-1, case["groups"], size).topk(min(2, size), 2).values.sum(2)
    allowed = torch.zeros_like(best).scatter_(1, best.topk(case["kept"], 1).indices, 1.0).repeat_interleave(size, 1)
    idx = c.masked_fill(allowed == 0, -math.inf).topk(case["k"], 1).indices
    gate = s.gather(1, idx)
    if case["renorm"]:
        gate = gate / gate.sum(1, keepdim=True)
    gate = gate * case["scale"]
    out = {"idx": idx.to(torch.int32), "gate": gate.detach(), "count": torch.bincount(idx.reshape(-1), minlength=case["M"]).to(torch.int32)}
    if case["mode"] == "step":
        out["dlogits"] = torch.autograd.grad(gate, logits, st["dgate"].double())[0]
    return out


def _exact_ortho(u):
    """One matrix: each step is a x + b (x x^T) x + c (x x^T)^2 x, multiplied out from the right."""
    x = u / torch.linalg.matrix_norm(u)
    a, b, c = COEF
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            g = x @ x.T
            once = g @ x
            twice = g @ once
        else:
            g = x.T @ x
            once = x @ g
            twice = once @ g
        x = a * x + b * once + c * twice
    return x


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, st)
    if case["op"] == "router":
        return _exact_router(case, st)
    if case["op"] == "ortho":
        return {"out": torch.stack([_exact_ortho(u.double()) for u in st["src"]])}
    out = {"param": st["param"].double(), "master": st["master"].double(), "m": []}
    at = st["at"].tolist()
    for i in range(case["trainable"]):
        g, m = st["grad"][i].double(), st["m"][i].double()
        m = BETA * m + g
        o = _exact_ortho(g + BETA * m if case["nesterov"] else m)
        w = out["master"][i]
        w -= case["lr"] * (DECAY * w + st["scale"] * o)
        out["param"][at[i]] = w
        out["m"].append(m)
    out["m"] = torch.stack(out["m"])
    return out
