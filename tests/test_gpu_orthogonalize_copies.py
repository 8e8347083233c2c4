"""Stacks whose matrices are copies of one another: the same bits wherever they stand."""
import numpy as np
import pytest
import torch

import paper_2602_11543_amd as S
from test_gpu_orthogonalize import TYPES, dt, matrices, run

pytestmark = pytest.mark.gpu


@TYPES
@pytest.mark.parametrize("n,rows,cols", [(70, 200, 328), (66, 130, 70), (130, 64, 64)])
def test_copies_of_a_matrix_get_the_same_bits(device, n, rows, cols, dtype):
    """Beyond the first launch of the optimizer step too, which updates 64 matrices."""
    one = matrices(1, rows, cols, 7)
    src = one.to(dtype).cuda().expand(n, rows, cols).contiguous()
    out = run(src)
    assert torch.equal(out, out[:1].expand_as(out))
    m, grad = one.cuda().expand(n, rows, cols).contiguous(), (one.flip(2) * 0.3).cuda().expand(n, rows, cols).contiguous()
    param = torch.full((n, rows, cols), 0.02, dtype=dtype, device="cuda")
    master = param.float()
    scratch = torch.empty(S.spes_orthogonalize_scratch_bytes(n, rows, cols, dt(dtype)), dtype=torch.uint8, device="cuda")
    S.spes_masked_muon(n, rows, cols, dt(dtype), param, np.ones(n, dtype=np.uint8), master, m, grad, 0.02, 0.9, 1, 0.1, 1.0, 5, None, 1.0, scratch)
    torch.cuda.synchronize()
    for t in (param, master, m):
        assert torch.equal(t, t[:1].expand_as(t))
