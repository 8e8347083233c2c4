"""One block around the expert layer on the device: the residual stream's addition and a root-mean-square norm, sigmoid routing in groups with a
steering bias, the routed SwiGLU experts, and the optimizer step that orthogonalises the experts' updates.  It holds the buffers and
makes the calls; the two products with the router's matrix are plain library products."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as S


class DeviceBlock:
    """Weights, state and buffers of one block for batches of T tokens.  `mask`: the experts that this node trains."""

    def __init__(self, T, d_model, n_experts, d_ff, top_k, mask, dtype="bf16", groups=1, kept_groups=1, scale=1.0, seed=0, device="cuda"):
        self.dt = S.SPES_F32 if dtype == "f32" else S.SPES_BF16
        self.T, self.d, self.M, self.f, self.k = T, d_model, n_experts, d_ff, top_k
        self.shape = S.moe_shape(T, d_model, n_experts, d_ff, top_k, self.dt, 0)
        self.opts = S.router_opts(S.SPES_SCORE_SIGMOID, groups, kept_groups, 1, scale)
        self.mask = np.asarray(mask, dtype=np.uint8)
        trainable = [e for e in range(n_experts) if self.mask[e]]
        n, st, f32 = len(trainable), S.torch_dtype(self.dt), torch.float32
        g = torch.Generator(device=device).manual_seed(seed)
        new = lambda *s, t=f32: torch.empty(*s, dtype=t, device=device)  # noqa: E731
        normal = lambda std, *s: (std * torch.randn(*s, device=device, generator=g)).to(st)  # noqa: E731
        self.norm_w = torch.ones(d_model, dtype=st, device=device)
        self.w_router = normal(d_model ** -0.5, n_experts, d_model)
        self.bias = torch.zeros(n_experts, dtype=f32, device=device)
        self.experts = {"gate": normal(d_model ** -0.5, n_experts, d_ff, d_model), "up": normal(d_model ** -0.5, n_experts, d_ff, d_model),
                        "down": normal(d_ff ** -0.5, n_experts, d_model, d_ff)}
        self.master = {k: w[trainable].float() for k, w in self.experts.items()}
        self.m = {k: torch.zeros_like(w) for k, w in self.master.items()}
        self.grad = {k: torch.zeros_like(w) for k, w in self.master.items()}
        # the shared matrices: AdamW, one "expert" each
        self.shared = {k: dict(master=w.float().clone(), m=torch.zeros(w.shape, device=device), v=torch.zeros(w.shape, device=device))
                       for k, w in (("norm_w", self.norm_w), ("w_router", self.w_router))}
        self.sum, self.h, self.y, self.out = (new(T, d_model, t=st) for _ in range(4))
        self.rstd = new(T)
        self.idx, self.gate, self.dgate = new(T, top_k, t=torch.int32), new(T, top_k), new(T, top_k)
        self.chosen, self.count = new(n_experts, t=torch.int32), new(n_experts, t=torch.int32)
        self.dlogits = new(T, n_experts)
        self.dh, self.dx = new(T, d_model, t=st), new(T, d_model, t=st)
        self.d_norm_w, self.d_w_router = torch.zeros(d_model, device=device), torch.zeros(n_experts, d_model, device=device)
        self.ctx = new(S.spes_moe_ctx_bytes(self.shape), t=torch.uint8)
        self.norm_scratch = new(S.spes_norm_scratch_bytes(T, d_model), t=torch.uint8)
        sides = ((d_ff, d_model), (d_model, d_ff))
        self.muon_scratch = new(max(S.spes_orthogonalize_scratch_bytes(n, r, c, self.dt) for r, c in sides), t=torch.uint8) if n else None
        self.steps = 0

    def forward(self, x, add):
        """x, add [T, d]: the stream and what the block before adds to it.  Returns the stream behind this block."""
        T, d = self.T, self.d
        S.spes_norm_fwd(S.SPES_NORM_RMS, T, d, self.dt, x, add, self.norm_w, None, 1e-6, self.sum, self.h, None, self.rstd)
        self.logits = self.h.float() @ self.w_router.float().t()
        S.spes_router_fwd(T, self.M, self.k, self.opts, self.logits, self.bias, self.idx, self.gate, self.chosen)
        S.spes_moe_fwd_routed(self.shape, self.h, self.idx, self.gate, *self.experts.values(), self.y, self.count, self.ctx)
        torch.add(self.sum, self.y, out=self.out)
        return self.out

    def backward(self, d_out, accumulate=0):
        """d_out [T, d]: gradient of the stream behind the block.  Returns that of the stream ahead of it, x's and add's alike."""
        T, d = self.T, self.d
        S.spes_moe_bwd_routed(self.shape, d_out, self.h, *self.experts.values(), self.ctx, self.mask, self.dh, self.dgate,
                              *(self.grad.values() if len(self.master["gate"]) else (None,) * 3), accumulate)
        S.spes_router_bwd(T, self.M, self.k, self.opts, self.logits, self.idx, self.dgate, self.dlogits)
        d_w_router = self.dlogits.t() @ self.h.float()
        self.d_w_router = self.d_w_router + d_w_router if accumulate else d_w_router          # (like the other gradients zeros ahead of the first batch)
        dh = (self.dh.float() + self.dlogits @ self.w_router.float()).to(self.dh.dtype)
        S.spes_norm_bwd(S.SPES_NORM_RMS, T, d, self.dt, dh, self.sum, self.norm_w, None, self.rstd, d_out, self.dx, self.d_norm_w, None, accumulate,
                        self.norm_scratch)
        return self.dx

    def step(self, lr=0.02, shared_lr=1e-3, weight_decay=0.1, bias_rate=1e-3):
        """Orthogonalised updates for the trained experts, AdamW for what every node trains; the bias moves towards an even load."""
        self.steps += 1
        for k, w in self.experts.items():
            rows, cols = w.shape[1:]
            S.spes_masked_muon(self.M, rows, cols, self.dt, w, self.mask, self.master[k], self.m[k], self.grad[k], lr, 0.95, 1, weight_decay,
                               0.2 * max(rows, cols) ** 0.5, 5, None, 1.0, self.muon_scratch)
        for k, grad in (("norm_w", self.d_norm_w), ("w_router", self.d_w_router)):
            w, s = getattr(self, k), self.shared[k]
            S.spes_masked_adamw(1, w.numel(), self.dt, w, np.ones(1, dtype=np.uint8), s["master"], s["m"], s["v"], grad.contiguous(), shared_lr, 0.9, 0.95,
                                1e-8, weight_decay, self.steps)
        load = self.chosen.float()
        self.bias += bias_rate * torch.sign(load.mean() - load)
