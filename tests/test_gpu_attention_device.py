"""Tensors of the attention half on another device than the current one are refused ahead of any launch."""
import pytest
import torch

import paper_2602_11543_amd as S
import test_gpu_attention
import test_gpu_qk_rope

pytestmark = pytest.mark.gpu


def test_another_device(monkeypatch):
    """(One device is enough to see it: the current one is said to be another.)"""
    p, r = test_gpu_attention.Problem([70, 33]), test_gpu_qk_rope.Problem(9)
    out, qk = p.forward(), r.forward()
    p.backward(**out), r.backward()
    torch.cuda.synchronize()
    stream = torch.cuda.current_stream().cuda_stream
    o, lse, scratch = torch.zeros_like(out["o"]), torch.zeros_like(out["lse"]), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    dq, dk, dv = (torch.zeros_like(t) for t in (p.q, p.k, p.v))
    q, k, dx = torch.zeros_like(qk[0]), torch.zeros_like(qk[1]), r.views(torch.zeros_like(r.qkv))
    at = torch._C._cuda_getDevice()
    calls = [lambda: S.spes_attn_fwd(p.shape(), p.q, p.k, p.v, p.q_start, p.k_start, None, o, lse, scratch, stream),
             lambda: S.spes_attn_bwd(p.shape(), p.d_o, p.q, p.k, p.v, p.q_start, p.k_start, None, out["o"], out["lse"], dq, dk, dv, scratch, stream),
             lambda: S.spes_qk_rope_fwd(r.shape(), r.q, r.k, r.qw, r.kw, r.table, r.pos, q, k, stream),
             lambda: S.spes_qk_rope_bwd(r.shape(), r.dq, r.dk, r.q, r.k, r.qw, r.kw, r.table, r.pos, *dx, None, None, 0, None, stream)]
    results = (o, lse, dq, dk, dv, q, k, *dx)
    with monkeypatch.context() as m:
        m.setattr(torch._C, "_cuda_getDevice", lambda: at + 1)
        for c in calls:
            with pytest.raises(S.SpesError, match="current device"):
                c()
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in results)
    for c in calls:
        c()
    torch.cuda.synchronize()
    assert all((t != 0).any() for t in results)
