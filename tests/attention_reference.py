"""Attention in 64 bits, sequence by sequence and head by head, with the allowances that its device form is held to.

An allowance counts roundings, each at most half a step (u = eps / 2 of its type) of what it rounds, w = 2^-24 for fp32:
  scores       a sum of D products in fp32 from bf16 or fp32 operands: at most (D + 8) w of the sum of magnitudes; as exponents, their product
               with log2 e, the difference to the maximum or lse and the exponential itself add 8 w of the magnitudes and of 1
  p            relative: that of its score, twice over (lse has it as well); rounded to the operands' type (bf16) ahead of the products
  o, dv        the sums over keys (rows) of p's errors times |v| (|do|), the sum itself at most (n + 64) w of its magnitudes, a rounding of the result
  delta        o's allowance and its own sum, weighted by |do|
  ds           p (dp - delta): p's relative error of it, p times the errors of dp and delta, rounded to the operands' type
  underflow    what fp32 (and bf16, whose exponents are the same) has below t = 2^-126 is nothing to the hardware's exponential and to its products: p and ds
               are off by t each, and so is a result, beside all of the above: with p = 10^-40 exact, the device has 0
  dq, dk       the sums over ds's errors times |k| (|q|), the sum itself, a rounding of the result
"""
import math

import torch

W = 2.0 ** -24
TINY = 2.0 ** -126


def seen(lq, lk, causal, window, device="cpu"):
    """[lq, lk]: which keys each query sees."""
    if not causal:
        return torch.ones(lq, lk, dtype=torch.bool, device=device)
    at = torch.arange(lq, device=device)[:, None] + (lk - lq)
    key = torch.arange(lk, device=device)[None, :]
    sees = key <= at
    return sees & (key > at - window) if window else sees


def head(q, k, v, scale, sees, u, d_o=None):
    """One head of one sequence: {name: (value, allowance)} in 64 bits.  u: half a step of the operands' type."""
    dtype_u = u if u > W else 0.0              # fp32 operands are not rounded
    lq, D = q.shape
    lk = k.shape[0]
    q, k, v = q.double(), k.double(), v.double()
    s, mag = scale * (q @ k.T), scale * (q.abs() @ k.abs().T)
    s = s.masked_fill(~sees, -math.inf)
    some = sees.any(1)
    lse = torch.logsumexp(s, 1) if lk else torch.full((lq,), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(some[:, None] & sees, torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
    top = mag.masked_fill(~sees, 0.0).amax(1) if lk else torch.zeros(lq, dtype=torch.float64, device=q.device)
    e_s = (D + 16) * W * top + 8 * W * (1 + torch.where(some, lse.abs(), 0.0))
    rel = (2 * e_s + 4 * W)[:, None]           # of p
    n = (max(lk, lq) + 64) * W
    out = {"lse": (lse, e_s + (lk + 16) * W)}
    o = p @ v
    o_allow = (rel + dtype_u + n) * (p @ v.abs()) + u * o.abs() + TINY * (1 + (sees.double() @ v.abs()))
    out["o"] = (o, o_allow)
    if d_o is None:
        return out
    d_o = d_o.double()
    dp = d_o @ v.T
    dp_allow = (D + 16) * W * (d_o.abs() @ v.abs().T)
    delta = (d_o * o).sum(1, keepdim=True)
    delta_allow = (d_o.abs() * o_allow).sum(1, keepdim=True) + (D + 16) * W * (d_o.abs() * o.abs()).sum(1, keepdim=True)
    ds = p * (dp - delta)
    # (the difference is of what dp and delta are, not of what is left of them)
    small = TINY * (1 + (dp - delta).abs()) * sees
    ds_allow = small + p * (dp_allow + delta_allow + 4 * W * (dp.abs() + delta.abs())) * (1 + rel) + ds.abs() * (rel + dtype_u)
    dv, dk, dq = p.T @ d_o, scale * (ds.T @ q), scale * (ds @ k)
    out["dv"] = (dv, (p * (rel + dtype_u + n)).T @ d_o.abs() + TINY * (1 + sees.double().T @ d_o.abs()))
    out["dk"] = (dk, scale * ((ds_allow + n * ds.abs()).T @ q.abs()) + TINY)
    out["dq"] = (dq, scale * ((ds_allow + n * ds.abs()) @ k.abs()) + (u + 4 * W) * dq.abs() + TINY)
    return out


def attention(q, k, v, seqs, scale, causal, window, d_o=None):
    """q [rows, H, D], k, v [krows, K, D]; seqs: (first query, queries, first key, keys).  {name: (value, allowance)}, NaN in rows of no sequence."""
    H, K, D = q.shape[1], k.shape[1], q.shape[2]
    u = torch.finfo(q.dtype).eps / 2
    new = lambda *size: torch.full(size, math.nan, dtype=torch.float64, device=q.device)  # noqa: E731
    out = {"o": (new(*q.shape), new(*q.shape)), "lse": (new(H, q.shape[0]), new(H, q.shape[0]))}
    if d_o is not None:
        out["dq"] = (new(*q.shape), new(*q.shape))
        out["dk"], out["dv"] = ((new(*k.shape), new(*k.shape)) for _ in range(2))
    for q0, lq, k0, lk in seqs:
        sees = seen(lq, lk, causal, window, q.device)
        rows, keys = slice(q0, q0 + lq), slice(k0, k0 + lk)
        if d_o is not None:
            for n in ("dk", "dv"):
                out[n][0][keys], out[n][1][keys] = 0.0, 0.0
        for h in range(H):
            c = h // (H // K)
            r = head(q[rows, h], k[keys, c], v[keys, c], scale, sees, u, None if d_o is None else d_o[rows, h])
            for n, (val, allow) in r.items():
                for i, x in enumerate((val, allow)):
                    if n == "lse":
                        out[n][i][h, rows] = x
                    elif n in ("o", "dq"):
                        out[n][i][rows, h] = x
                    else:
                        out[n][i][keys, c] += x
    if d_o is not None:
        for n in ("dk", "dv"):                 # the sum over heads, and one rounding of it
            out[n] = (out[n][0], out[n][1] + (u + 64 * W) * out[n][0].abs())
    return out


def excess(got, want, allow):
    """By how much the worst element is off beyond its allowance, and where; infinities have to be the same, rows of no sequence are skipped."""
    got = got.double()
    there = ~torch.isnan(want)
    inf = there & torch.isinf(want)
    if not torch.equal(got[inf], want[inf]):
        return math.inf, "infinities differ"
    there = there & ~inf
    if not there.any():
        return 0.0, ""
    if not torch.isfinite(got[there]).all():
        return math.inf, "not finite"
    over = ((got - want).abs() - allow)[there]
    return float(over.max()), f"error up to {float((got - want).abs()[there].max()):.3g}, allowance there {float(allow[there][over.argmax()]):.3g}"
