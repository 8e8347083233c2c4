"""The attention half of a block as a training program and its evaluation call it, as a list of cases that can be timed and compared.

    qk       queries and keys ahead of attention: the norm of every head and the rotation by the token's position, read out of the
             projection's output: `forward` alone, or a `step` with the gradients of the projection's output and of the norm's weights
    attn     attention over sequences of unequal length, heads that share keys, causal or not, within a window or not: `forward` (also one
             token against a long cache), or a `step` with the gradients of queries, keys and values

Each case is one pass through the public entry points (`own`), or the same in elementary operations in 32 bits.  Shapes follow the
repository's own layer workloads: widths of 768, 2048 and 4096 as heads of 64 and 128, their tokens and micro-batches, and sizes around them.
"""
import math

import torch

own = False

EPS, BASE = 1e-6, 10000.0


def _qk(name, mode, T, heads, kv, dim, rot, interleaved, dtype, norm, lens, far=0):
    """lens: the documents that the tokens belong to; positions count from `far` in each."""
    return dict(name=name, op="qk", mode=mode, T=T, heads=heads, kv=kv, dim=dim, rot=rot, interleaved=interleaved, dtype=dtype, norm=norm, lens=lens, far=far)


def _attn(name, mode, lens, keys, room, heads, kv, dim, dtype, causal, window, packed):
    """lens: queries of each sequence; keys: its keys, the same where empty; room: rows of a sequence in the cache, 0 where sequences stand one
    behind the other; packed: the values are read where the projection wrote them."""
    return dict(name=name, op="attn", mode=mode, lens=lens, keys=keys, room=room, heads=heads, kv=kv, dim=dim, dtype=dtype, causal=causal, window=window,
                packed=packed)


def _text(lens):
    return ",".join(str(n) for n in lens)


def _numbers(text):
    return [int(n) for n in text.split(",")]


# documents in one training batch of 16384 tokens: many short ones, a few long ones
DOCUMENTS = (6011, 3500, 2049, 1777, 1024, 640, 511, 300, 256, 129, 77, 64, 31, 8, 6, 1)
# how far the sequences of a serving batch have come
CACHED = (8192, 7001, 6400, 5555, 4097, 4096, 3333, 2900, 2500, 2048, 1999, 1500, 1024, 1001, 777, 640, 512, 511, 400, 300, 257, 255, 192, 129, 100, 77, 64, 33,
          17, 9, 2, 1)


def listed():
    return [
        # a serving step of 32 sequences far into their contexts: where a launch's latency is what counts
        _qk("qk_decode", "forward", 32, 16, 4, 128, 128, False, "bf16", True, _text([1] * 32), 100000),
        # a micro-batch of 2 x 2048 tokens of the smallest training workload
        _qk("qk_paper_1b", "step", 4096, 12, 12, 64, 64, False, "bf16", True, _text([2048] * 2)),
        # full precision, a head that is no power of two, only its first part rotated, neighbours as pairs
        _qk("qk_ragged_f32", "step", 1531, 10, 5, 80, 64, True, "f32", True, _text([1000, 530, 1])),
        # the widest training workload
        _qk("qk_cfg3", "step", 32768, 32, 8, 128, 128, False, "bf16", True, _text([4096] * 8)),
        # scoring one short sequence
        _attn("attn_score_short", "forward", "200", "", 0, 12, 12, 64, "bf16", True, 0, True),
        # the next 512 tokens of a long prompt, behind 15488 that the cache holds
        _attn("attn_chunk", "forward", "512", "16000", 0, 32, 8, 128, "bf16", True, 0, False),
        # a serving step: one token each of 32 sequences, in a cache with room for 8192
        _attn("attn_decode", "forward", _text([1] * 32), _text(CACHED), 8192, 32, 8, 128, "bf16", True, 0, False),
        # one token against a single long context
        _attn("attn_decode_long", "forward", "1", "131071", 131072, 16, 4, 128, "bf16", True, 0, False),
        # a micro-batch of the smallest training workload
        _attn("attn_paper_1b", "step", _text([2048] * 2), "", 0, 12, 12, 64, "bf16", True, 0, True),
        # documents packed into one batch
        _attn("attn_documents", "step", _text(DOCUMENTS), "", 0, 16, 4, 128, "bf16", True, 0, True),
        # full precision, a head that is no power of two, a window
        _attn("attn_ragged_f32", "step", _text([1001, 1500, 259]), "", 0, 10, 5, 80, "f32", True, 700, False),
        # the widest training workload
        _attn("attn_cfg3", "step", _text([4096] * 8), "", 0, 32, 8, 128, "bf16", True, 0, True),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)


def _split(rng, total):
    """Documents that fill `total` tokens."""
    lens = []
    while total > 0:
        n = min(total, _log(rng, 1, 8192))
        lens.append(n)
        total -= n
        if len(lens) == 24 and total > 0:
            lens[-1] += min(total, 8192)
            total = 0
    return lens


def draw(rng):
    """Another case of the same ranges: 1 to 32768 tokens with 1 to 32 heads of 32 to 128 (256 ahead of attention), sequences of 1 to 8192
    queries and up to 131072 keys."""
    op = rng.choice(["qk", "attn", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 3, 4, 5, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4])
    if op == "qk":
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 160, 256])
        lens = _split(rng, _log(rng, 1, 32768))
        return dict(op=op, mode=rng.choice(["forward", "step", "step"]), T=sum(lens), heads=heads, kv=kv, dim=dim,
                    rot=rng.choice([dim, dim, 16 * rng.randint(1, dim // 16)]), interleaved=rng.random() < 0.4, dtype=dtype, norm=rng.random() < 0.8,
                    lens=_text(lens), far=rng.choice([0, 0, _log(rng, 1000, 100000)]))
    dim = rng.choice([32, 64, 64, 72, 80, 96, 112, 128, 128, 128])
    kind = rng.choice(["forward", "step", "step", "decode"])
    while True:
        window, causal = 0, True
        if kind == "decode":
            lens = [rng.choice([1, 1, 1, rng.randint(1, 8)])] * rng.choice([1, 1, 2, 4, 8, 16, 32])
            keys = [max(lens[0], _log(rng, 1, 131072)) for _ in lens]
            if rng.random() < 0.2:
                window = _log(rng, 16, 8192)
            room = rng.choice([0, max(keys)])
            rows = room * len(lens) if room else sum(keys)
            if rows * kv * dim > 32 * 8192 * 8 * 128:
                continue
            return dict(op=op, mode="forward", lens=_text(lens), keys=_text(keys), room=room, heads=heads, kv=kv, dim=dim, dtype=dtype, causal=True, window=window,
                        packed=False)
        lens = _split(rng, _log(rng, 16, 32768))
        keys = ""
        if kind == "forward" and rng.random() < 0.5:
            keys = _text([n + rng.choice([0, _log(rng, 1, 4096)]) for n in lens])
        form = rng.random()
        if form < 0.2:
            causal = False
        elif form < 0.4:
            window = _log(rng, 16, 4096)
        case = dict(op=op, mode=kind, lens=_text(lens), keys=keys, room=0, heads=heads, kv=kv, dim=dim, dtype=dtype, causal=causal, window=window,
                    packed=keys == "" and rng.random() < 0.5)
        if work(case)["flops"] * (8 if dtype == "f32" else 1) <= 3.85e12:
            return case


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *size: torch.randn(*size, device="cuda", generator=g)  # noqa: E731
    t, H, K, D = _type(case), case["heads"], case["kv"], case["dim"]
    st = {"case": case, "lens": _numbers(case["lens"])}
    if case["op"] == "qk":
        T, rot = case["T"], case["rot"]
        # the projection's output: features of unequal size
        st["qkv"] = (normal(T, (H + 2 * K) * D) * (0.5 + torch.rand((H + 2 * K) * D, device="cuda", generator=g))).to(t)
        st["q"], st["k"] = st["qkv"][:, : H * D].view(T, H, D), st["qkv"][:, H * D: (H + K) * D].view(T, K, D)
        st["q_weight"], st["k_weight"] = ((1 + 0.1 * normal(D)).to(t) for _ in range(2)) if case["norm"] else (None, None)
        st["pos"] = torch.cat([case["far"] + torch.arange(n, device="cuda") for n in st["lens"]]).to(torch.int32)
        n_pos = case["far"] + max(st["lens"])
        angle = torch.arange(n_pos, device="cuda").double()[:, None] * BASE ** (-2.0 / rot * torch.arange(rot // 2, device="cuda").double())
        st["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        if case["mode"] == "step":
            st["dq"], st["dk"] = normal(T, H, D).to(t), normal(T, K, D).to(t)
        return st
    lens = st["lens"]
    keys = st["keys"] = _numbers(case["keys"]) if case["keys"] else lens
    rows, krows = sum(lens), case["room"] * len(lens) if case["room"] else sum(keys)
    # heads that differ in how sharply they look, and a first key that draws all of them
    st["q"] = (normal(rows, H, D) * (0.5 + torch.rand(H, 1, device="cuda", generator=g))).to(t)
    k = normal(krows, K, D)
    st["k_at"] = [i * case["room"] for i in range(len(keys))] if case["room"] else _starts(keys)[:-1]
    first = [at for at, n in zip(st["k_at"], keys) if n > 0]
    k[first] += 0.5 * normal(1, K, D)
    st["k"] = k.to(t)
    if case["packed"]:
        st["qkv"] = normal(rows, (H + 2 * K) * D).to(t)
        st["v"] = st["qkv"][:, (H + K) * D:].view(rows, K, D)
    else:
        st["v"] = normal(krows, K, D).to(t)
    st["q_start"] = _ints(_starts(lens))
    if case["room"]:
        st["k_start"], st["k_len"] = _ints(st["k_at"] + [krows]), _ints(keys)
    else:
        st["k_start"], st["k_len"] = _ints(_starts(keys)), None
    if case["mode"] == "step":
        st["do"] = normal(rows, H, D).to(t)
    return st


# ---- the plain forms ----


def _turn(x, cos, sin, interleaved):
    """x [T, heads, rot]; cos, sin [T, 1, rot / 2]"""
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).reshape(x.shape)
    a, b = x[..., : x.shape[2] // 2], x[..., x.shape[2] // 2:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], 2)


def _plain_qk(case, st):
    t, rot, out = _type(case), case["rot"], {}
    cs = st["table"][st["pos"].long()]
    cos, sin = cs[:, None, : rot // 2], cs[:, None, rot // 2:]
    for n in ("q", "k"):
        x = st[n].float()
        if case["norm"]:
            w = st[n + "_weight"].float()
            rstd = 1.0 / torch.sqrt((x * x).mean(2, keepdim=True) + EPS)
            hat = x * rstd
            y = hat * w
        else:
            y = x
        out[n] = torch.cat([_turn(y[..., :rot], cos, sin, case["interleaved"]), y[..., rot:]], 2).to(t)
        if case["mode"] == "step":
            dy = st["d" + n].float()
            dy = torch.cat([_turn(dy[..., :rot], cos, -sin, case["interleaved"]), dy[..., rot:]], 2)
            if case["norm"]:
                out["d_" + n + "_weight"] = (dy * hat).sum((0, 1))
                h = dy * w
                dy = (h - hat * (h * hat).mean(2, keepdim=True)) * rstd
            out["d" + n] = dy.to(t)
    return out


def _hidden(case, first, n, lq, lk):
    """[n, lk]: keys that queries first .. first + n of lq do not see; None where they see all."""
    if not case["causal"]:
        return None
    at = torch.arange(first, first + n, device="cuda")[:, None] + (lk - lq)
    key = torch.arange(lk, device="cuda")[None, :]
    hidden = key > at
    return hidden | (key <= at - case["window"]) if case["window"] else hidden


def _pieces(lq, lk, heads, limit):
    """Ranges of queries whose scores over the keys are at most `limit` values."""
    n = max(1, min(lq, limit // max(1, lk * heads)))
    return [(i, min(n, lq - i)) for i in range(0, lq, n)]


def _plain_attn(case, st):
    H, K, D, t = case["heads"], case["kv"], case["dim"], _type(case)
    G, scale = H // K, 1.0 / math.sqrt(D)
    q, k, v = st["q"], st["k"], st["v"]
    out = {"o": torch.empty_like(q), "lse": torch.empty(H, q.shape[0], device="cuda")}
    step = case["mode"] == "step"
    if step:
        out["dq"], out["dk"], out["dv"] = torch.empty_like(q), torch.zeros(k.shape, dtype=t, device="cuda"), torch.zeros(k.shape, dtype=t, device="cuda")
    at = 0
    for lq, lk, kat in zip(st["lens"], st["keys"], st["k_at"]):
        kf, vf = k[kat: kat + lk].float().transpose(0, 1).contiguous(), v[kat: kat + lk].float().transpose(0, 1).contiguous()      # [K, lk, D]
        dk, dv = torch.zeros_like(kf), torch.zeros_like(vf)
        for first, n in _pieces(lq, lk, H, 1 << 30):
            rows = slice(at + first, at + first + n)
            heads = lambda x: x[rows].float().view(n, K, G, D).permute(1, 2, 0, 3).reshape(K, G * n, D)  # noqa: E731
            back = lambda x: x.view(K, G, n, D).permute(2, 0, 1, 3).reshape(n, H, D)  # noqa: E731
            qf = heads(q) * scale
            s = torch.bmm(qf, kf.transpose(1, 2).contiguous())
            hidden = _hidden(case, first, n, lq, lk)
            if hidden is not None:
                s = s.view(K, G, n, lk).masked_fill(hidden, -math.inf).view(K, G * n, lk)
            top = s.amax(2, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(2, keepdim=True)
            p = p / total
            of = torch.bmm(p, vf)
            out["o"][rows] = back(of).to(t)
            out["lse"][:, rows] = (top + torch.log(total)).view(H, n)
            if step:
                do = heads(st["do"])
                dv += torch.bmm(p.transpose(1, 2).contiguous(), do)
                dp = torch.bmm(do, vf.transpose(1, 2).contiguous())
                ds = p * (dp - (do * of).sum(2, keepdim=True))
                out["dq"][rows] = back(torch.bmm(ds, kf) * scale).to(t)
                dk += torch.bmm(ds.transpose(1, 2).contiguous(), qf)
        if step:
            out["dk"][kat: kat + lk], out["dv"][kat: kat + lk] = dk.transpose(0, 1).to(t), dv.transpose(0, 1).to(t)
        at += lq
    return out


# ---- the framework's calls ----


def _kept(st, name, make):
    """A buffer that the program makes once and keeps."""
    if name not in st:
        st[name] = make()
    return st[name]


def _own(st):
    import paper_2602_11543_amd as S

    case = st["case"]
    dt = S.SPES_F32 if case["dtype"] == "f32" else S.SPES_BF16
    step, D = case["mode"] == "step", case["dim"]
    scratch = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    if case["op"] == "qk":
        def make():
            shape = S.qk_shape(case["T"], case["heads"], case["kv"], D, case["rot"], dt, int(case["interleaved"]), st["table"].shape[0], EPS)
            o = {n: torch.empty(st[n].shape, dtype=st[n].dtype, device="cuda") for n in ("q", "k")}
            if step:
                grad = torch.empty_like(st["qkv"])      # of the projection's output; attention writes the values' part
                H, K = case["heads"], case["kv"]
                o["dq"], o["dk"] = grad[:, : H * D].view(-1, H, D), grad[:, H * D: (H + K) * D].view(-1, K, D)
                if case["norm"]:
                    o["d_q_weight"], o["d_k_weight"] = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
            return shape, o, scratch(S.spes_qk_rope_scratch_bytes(shape)) if step else None

        shape, o, buf = _kept(st, "out", make)
        S.spes_qk_rope_fwd(shape, st["q"], st["k"], st["q_weight"], st["k_weight"], st["table"], st["pos"], o["q"], o["k"])
        if step:
            S.spes_qk_rope_bwd(shape, st["dq"], st["dk"], st["q"], st["k"], st["q_weight"], st["k_weight"], st["table"], st["pos"], o["dq"], o["dk"],
                               o.get("d_q_weight"), o.get("d_k_weight"), 0, buf)
        return o

    def make():
        q, k = st["q"], st["k"]
        shape = S.attn_shape(len(st["lens"]), q.shape[0], k.shape[0], case["heads"], case["kv"], D, dt, int(case["causal"]), case["window"], 1.0 / math.sqrt(D))
        o = {"o": torch.empty_like(q), "lse": torch.empty(case["heads"], q.shape[0], device="cuda")}
        if step:
            o["dq"], o["dk"] = torch.empty_like(q), torch.empty_like(k)
            o["dv"] = torch.empty_like(st["qkv"])[:, -k.shape[1] * D:].view(k.shape) if case["packed"] else torch.empty_like(k)
        return shape, o, scratch(max(S.spes_attn_scratch_bytes(shape, b) for b in range(1 + step)))

    shape, o, buf = _kept(st, "out", make)
    S.spes_attn_fwd(shape, st["q"], st["k"], st["v"], st["q_start"], st["k_start"], st["k_len"], o["o"], o["lse"], buf)
    if step:
        S.spes_attn_bwd(shape, st["do"], st["q"], st["k"], st["v"], st["q_start"], st["k_start"], st["k_len"], o["o"], o["lse"], o["dq"], o["dk"], o["dv"], buf)
    return o


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    return _plain_qk(case, state) if case["op"] == "qk" else _plain_attn(case, state)


def _seen(case):
    """Pairs of a query and a key that it sees."""
    lens = _numbers(case["lens"])
    pairs = 0
    for lq, lk in zip(lens, _numbers(case["keys"]) if case["keys"] else lens):
        if not case["causal"]:
            pairs += lq * lk
            continue
        pairs += sum(min(at + 1, case["window"] or at + 1) for at in range(lk - lq, lk) if at >= 0)
    return pairs


def work(case):
    """Every input once, every output once; a key that no query sees is not read, a pair that is hidden costs nothing."""
    es, step = 4 if case["dtype"] == "f32" else 2, case["mode"] == "step"
    H, K, D = case["heads"], case["kv"], case["dim"]
    if case["op"] == "qk":
        n = case["T"] * (H + K) * D
        return {"bytes": n * es * (4 if step else 2) + case["T"] * (4 + 4 * case["rot"]), "flops": n * (20 if step else 8)}
    lens = _numbers(case["lens"])
    keys = _numbers(case["keys"]) if case["keys"] else lens
    rows = sum(lens)
    krows = sum(min(lk, lq - 1 + case["window"]) if case["window"] else lk for lq, lk in zip(lens, keys))
    moved = (2 * rows * H + 2 * krows * K) * D * es + rows * H * 4
    if step:
        moved += (2 * rows * H + 2 * krows * K) * D * es
    return {"bytes": moved, "flops": _seen(case) * H * D * (14 if step else 4)}


# ---- the definitions in 64 bits ----


def _exact_qk(case, st):
    T, D, rot, out = case["T"], case["dim"], case["rot"], {}
    pairs = torch.arange(rot // 2, device="cuda")
    turn = torch.exp(1j * st["pos"].double()[:, None] * BASE ** (-2.0 * pairs.double() / rot))[:, None, :]
    first, second = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + rot // 2)
    for n in ("q", "k"):
        x = st[n].double().requires_grad_(True)
        leaves, y = [x], x
        if case["norm"]:
            w = st[n + "_weight"].double().requires_grad_(True)
            leaves.append(w)
            y = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.index_copy(2, first, z.real).index_copy(2, second, z.imag)
        out[n] = y.detach()
        if case["mode"] == "step":
            grads = torch.autograd.grad(y, leaves, st["d" + n].double())
            out["d" + n] = grads[0]
            if case["norm"]:
                out["d_" + n + "_weight"] = grads[1]
    return out


def _exact_attn(case, st):
    H, K, D = case["heads"], case["kv"], case["dim"]
    G, step = H // K, case["mode"] == "step"
    q, k, v = (st[n].double() for n in ("q", "k", "v"))
    out = {"o": torch.empty_like(q), "lse": torch.empty(H, q.shape[0], device="cuda", dtype=torch.float64)}
    if step:
        out.update(dq=torch.empty_like(q), dk=torch.zeros(k.shape, device="cuda", dtype=torch.float64), dv=torch.zeros(k.shape, device="cuda", dtype=torch.float64))
    at = 0
    for lq, lk, kat in zip(st["lens"], st["keys"], st["k_at"]):
        for h in range(H):
            kh, vh = k[kat: kat + lk, h // G], v[kat: kat + lk, h // G]
            for first, n in _pieces(lq, lk, 1, 1 << 28):
                rows = slice(at + first, at + first + n)
                s = (q[rows, h] @ kh.T) / math.sqrt(D)
                hidden = _hidden(case, first, n, lq, lk)
                if hidden is not None:
                    s.masked_fill_(hidden, -math.inf)
                out["lse"][h, rows] = torch.logsumexp(s, 1)
                p = torch.softmax(s, 1)
                del s
                out["o"][rows, h] = p @ vh
                if step:
                    do = st["do"][rows, h].double()
                    out["dv"][kat: kat + lk, h // G] += p.T @ do
                    dp = do @ vh.T
                    dp -= (p * dp).sum(1, keepdim=True)
                    dp *= p
                    del p
                    out["dq"][rows, h] = (dp @ kh) / math.sqrt(D)
                    out["dk"][kat: kat + lk, h // G] += (dp.T @ q[rows, h]) / math.sqrt(D)
        at += lq
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_qk(case, st) if case["op"] == "qk" else _exact_attn(case, st)
