"""Streams that the Infinity Cache does not hold, which kernels of their own read and write past it: results as everywhere else."""
import numpy as np
import pytest
import torch

import test_gpu_norm as N
import test_gpu_orthogonalize as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [N.LAYER, N.RMS], ids=["layer", "rms"])
@pytest.mark.parametrize("rows,cols,dtype", [(32768, 2048, torch.bfloat16), (20000, 2048, torch.float32), (8200, 8192, torch.bfloat16)])
def test_norm(device, rows, cols, dtype, kind):
    i = N.inputs(rows, cols, dtype, kind, True, False, 1)
    N.check(kind, i, 1e-5, N.run(kind, i, 1e-5))


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("rows,cols", [(1024, 4096), (4096, 1000)])
def test_optimizer_step(device, rows, cols, nesterov):
    mask = np.ones(11, dtype=np.uint8)
    mask[4] = 0
    O.muon(device, torch.bfloat16, 11, mask, rows, cols, nesterov, check=(0, 9))


@pytest.mark.parametrize("n,dtype", [(33, torch.bfloat16), (17, torch.float32)])
def test_orthogonalisation(device, n, dtype):
    src = O.matrices(n, 1024, 4096, 2).to(dtype).cuda()
    out = O.run(src)
    for i in (0, n - 1):
        O.near(out[i], O.exact(src[i]), O.out_allow(dtype))
