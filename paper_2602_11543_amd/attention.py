"""The attention half of a block on the device: root-mean-square norm, projections, norm of queries' and keys' heads with the rotation by position, and causal
attention over sequences of unequal length, forward and backward, with the optimizer step; and single tokens against a cache.  It holds the buffers and
makes the calls; the products with the projections' matrices are plain library products."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as S


def rotation_table(n_pos, rot_dim, base=10000.0, device="cuda"):
    """Cosines and sines of every position's angles, formed in 64 bits: [n_pos, rot_dim] as spes_qk_rope_fwd takes them."""
    pair = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
    angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * base ** (-2.0 / rot_dim * pair)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


class DeviceAttention:
    """Weights, state and buffers for batches of T tokens.  Every node trains these matrices.  rot_dim: elements of a head that are rotated, all of them if
    not given, 0 for none."""

    def __init__(self, T, d_model, heads, kv_heads, head_dim, n_pos, dtype="bf16", rot_dim=None, window=0, seed=0, device="cuda"):
        self.dt = S.SPES_F32 if dtype == "f32" else S.SPES_BF16
        self.T, self.d, self.H, self.K, self.D, self.window, self.n_pos = T, d_model, heads, kv_heads, head_dim, window, n_pos
        self.rot = head_dim if rot_dim is None else rot_dim
        st, f32 = S.torch_dtype(self.dt), torch.float32
        g = torch.Generator(device=device).manual_seed(seed)
        new = lambda *s, t=f32: torch.empty(*s, dtype=t, device=device)  # noqa: E731
        normal = lambda std, *s: (std * torch.randn(*s, device=device, generator=g)).to(st)  # noqa: E731
        width = (heads + 2 * kv_heads) * head_dim
        self.w = {"norm": torch.ones(d_model, dtype=st, device=device), "qkv": normal(d_model ** -0.5, width, d_model),
                  "q": torch.ones(head_dim, dtype=st, device=device), "k": torch.ones(head_dim, dtype=st, device=device),
                  "o": normal((heads * head_dim) ** -0.5, d_model, heads * head_dim)}
        self.state = {n: dict(master=w.float().clone(), m=torch.zeros(w.shape, device=device), v=torch.zeros(w.shape, device=device)) for n, w in self.w.items()}
        self.grad = {n: torch.zeros(w.shape, device=device) for n, w in self.w.items()}
        self.table = rotation_table(n_pos, self.rot, device=device) if self.rot else None
        self.h, self.rstd, self.dx = new(T, d_model, t=st), new(T), new(T, d_model, t=st)
        self.q, self.k = new(T, heads, head_dim, t=st), new(T, kv_heads, head_dim, t=st)
        self.d_heads = new(T * (heads + kv_heads) * head_dim, t=st)          # of q and k, one behind the other, so that one call clears both
        self.dq, self.dk = self.d_heads[: self.q.numel()].view_as(self.q), self.d_heads[self.q.numel():].view_as(self.k)
        self.o, self.lse = torch.empty_like(self.q), new(heads, T)
        self.qkv, self.d_qkv = new(T, width, t=st), new(T, width, t=st)
        self.qk = S.qk_shape(T, heads, kv_heads, head_dim, self.rot, self.dt, 0, n_pos)
        self.norm_scratch = new(S.spes_norm_scratch_bytes(T, d_model), t=torch.uint8)
        self.qk_scratch = new(S.spes_qk_rope_scratch_bytes(self.qk), t=torch.uint8)
        self.steps, self.cache, self.scratch = 0, None, {}

    def _heads(self, t):
        """Views of a projection's output, or of its gradient: queries, keys, values."""
        H, K, D = self.H, self.K, self.D
        return t[:, : H * D].view(-1, H, D), t[:, H * D: (H + K) * D].view(-1, K, D), t[:, (H + K) * D:].view(-1, K, D)

    def _shape(self, starts):
        return S.attn_shape(starts.numel() - 1, self.T, self.T, self.H, self.K, self.D, self.dt, 1, self.window)

    def _scratch(self, shape, backward, use="batch"):
        """Scratch for the call.  Captured graphs have the addresses of what was handed out, so a buffer that is outgrown is kept; each is twice the one
        before at least, and those kept are not more than the newest one.  Single tokens have their own, which batches do not grow."""
        need, kept = S.spes_attn_scratch_bytes(shape, backward), self.scratch.setdefault(use, [])
        if not kept or kept[-1].numel() < need:
            kept.append(torch.empty(max(need, 2 * kept[-1].numel() if kept else 0), dtype=torch.uint8, device=self.h.device))
        return kept[-1]

    def forward(self, x, starts, pos):
        """x [T, d]: the stream; starts [n + 1] i32: where its sequences begin, and the last one's end; pos [T] i32: a token's place in its
        sequence.  Rows ahead of the first sequence and behind the last one (finite, with a place that the table has) get nothing added and add nothing to
        the gradients.  Returns what this half adds to the stream.  A caller that captures the calls into a graph makes one eager call first, which
        takes the scratch."""
        T, d = self.T, self.d
        S.spes_norm_fwd(S.SPES_NORM_RMS, T, d, self.dt, x, None, self.w["norm"], None, 1e-6, None, self.h, None, self.rstd)
        torch.mm(self.h, self.w["qkv"].t(), out=self.qkv)
        q, k, v = self._heads(self.qkv)
        S.spes_qk_rope_fwd(self.qk, q, k, self.w["q"], self.w["k"], self.table, pos if self.rot else None, self.q, self.k)
        shape = self._shape(starts)
        # (attention leaves rows of no sequence as they are, and the products below go over all rows.  Cleared whole: which rows these are is known on the
        # device alone; 32768 rows of 32 / 8 heads of 128 in bf16, o and the three gradients, 0.7 GB to write)
        self.o.zero_()
        S.spes_attn_fwd(shape, self.q, self.k, v, starts, starts, None, self.o, self.lse, self._scratch(shape, 0))
        return self.o.view(T, -1) @ self.w["o"].t()

    def backward(self, d_add, x, starts, pos, d_stream=None, accumulate=0):
        """d_add [T, d]: gradient of what the last forward returned, x, starts and pos as they were for that; d_stream: the one that reaches x along the
        stream.  Returns x's."""
        T, d = self.T, self.d

        def product(name, a, b):               # (into the gradient's own place: graphs and the optimizer step know it by that)
            if accumulate:
                self.grad[name] += a.float().t() @ b.float()
            else:
                torch.mm(a.float().t(), b.float(), out=self.grad[name])

        product("o", d_add, self.o.view(T, -1))
        d_o = (d_add @ self.w["o"]).view(T, self.H, self.D)
        q, k, v = self._heads(self.qkv)
        dq, dk, dv = self._heads(self.d_qkv)
        self.d_heads.zero_()
        dv.zero_()
        shape = self._shape(starts)
        S.spes_attn_bwd(shape, d_o, self.q, self.k, v, starts, starts, None, self.o, self.lse, self.dq, self.dk, dv, self._scratch(shape, 1))
        S.spes_qk_rope_bwd(self.qk, self.dq, self.dk, q, k, self.w["q"], self.w["k"], self.table, pos if self.rot else None, dq, dk, self.grad["q"], self.grad["k"],
                           accumulate, self.qk_scratch)
        product("qkv", self.d_qkv, self.h)
        dh = self.d_qkv @ self.w["qkv"]
        S.spes_norm_bwd(S.SPES_NORM_RMS, T, d, self.dt, dh, x, self.w["norm"], None, self.rstd, d_stream, self.dx, self.grad["norm"], None, accumulate,
                        self.norm_scratch)
        return self.dx

    def step(self, lr=1e-3, weight_decay=0.1):
        self.steps += 1
        for n, w in self.w.items():
            s = self.state[n]
            S.spes_masked_adamw(1, w.numel(), self.dt, w, np.ones(1, dtype=np.uint8), s["master"], s["m"], s["v"], self.grad[n].contiguous(), lr, 0.9, 0.95, 1e-8,
                                weight_decay if w.dim() > 1 else 0.0, self.steps)

    def start_cache(self, n_seq, room):
        """Empty caches with room for `room` tokens of each of n_seq sequences.  Caches of these sizes that are there already are emptied where they are, and
        graphs that captured decode() go on with them; with others such graphs are not to be replayed any more."""
        dev, st = self.h.device, S.torch_dtype(self.dt)
        if n_seq < 0 or room < 0 or n_seq * room > 2 ** 31 - 2 ** 16:          # (as many rows as spes_attn_fwd takes)
            raise S.SpesError("start_cache: more rows than a cache can have")
        row0 = torch.arange(n_seq, dtype=torch.int32, device=dev) * room
        self.taken = 0
        if self.cache is not None and self.cache[0].shape[:2] == (n_seq, room):
            self.length.zero_()
            self.next.copy_(row0)
            return
        self.room, self.limit = room, min(room, self.n_pos)
        # one row more than there is room for takes what does not fit
        self.rows = [torch.empty(n_seq * room + 1, self.K, self.D, dtype=st, device=dev) for _ in range(2)]
        self.cache = [c[:-1].view(n_seq, room, self.K, self.D) for c in self.rows]
        self.length = torch.zeros(n_seq, dtype=torch.int32, device=dev)
        self.row0, self.next, self.spare = row0, row0.long(), torch.full((n_seq,), n_seq * room, dtype=torch.int64, device=dev)
        self.q_start = torch.arange(n_seq + 1, dtype=torch.int32, device=dev)

    def decode(self, x):
        """x [n_seq, d]: each sequence's next token.  Its keys and values join the cache; returns what this half adds to the stream.  A call may be captured into a
        graph, behind an eager one, which takes the scratch.  Where replays, which the host does not count, go on beyond the room or the
        positions, what they return is NaN and the caches stay as they are."""
        n, H, K, D = x.shape[0], self.H, self.K, self.D
        if self.cache is None or n != self.cache[0].shape[0] or self.taken >= self.limit:
            raise S.SpesError("decode: no cache for this many sequences, or its room or the positions are used up")
        new = lambda *s, t=x.dtype: torch.empty(*s, dtype=t, device=x.device)  # noqa: E731
        h, q, k, o = new(n, self.d), new(n, H, D), new(n, K, D), new(n, H, D)
        S.spes_norm_fwd(S.SPES_NORM_RMS, n, self.d, self.dt, x, None, self.w["norm"], None, 1e-6, None, h, None, new(n, t=torch.float32))
        qp, kp, vp = self._heads(h @ self.w["qkv"].t())
        # (a position beyond the limit is none of the table's, and gives NaN)
        S.spes_qk_rope_fwd(S.qk_shape(n, H, K, D, self.rot, self.dt, 0, self.limit), qp, kp, self.w["q"], self.w["k"], self.table,
                           self.length if self.rot else None, q, k)
        fits = self.length < self.limit
        if not self.rot:
            q.masked_fill_(~fits[:, None, None], float("nan"))
        at = torch.where(fits, self.next, self.spare)
        for c, t in zip(self.rows, (k, vp)):
            c.index_copy_(0, at, t)
        self.length += 1
        self.next += 1
        shape = S.attn_shape(n, n, n * self.room, H, K, D, self.dt, 1, self.window)
        S.spes_attn_fwd(shape, q, *(c.view(-1, K, D) for c in self.cache), self.q_start, self.row0, self.length, o, new(H, n, t=torch.float32),
                        self._scratch(shape, 0, "tokens"))
        if not torch.cuda.is_current_stream_capturing():
            self.taken += 1
        return o.view(n, -1) @ self.w["o"].t()
