"""How close the GELU of bf16 results is, value by value: the product is zero and the bias is z.

Tolerance: half a bf16 step (2^-8 of the value at most); up to |z| = 6 the evaluation's 8e-6 of the value (6.6e-6 of the fit in fp32
arithmetic and a step of the exponential, 1.2e-7); beyond, 5e-14 (4.1e-14 of the fit).  Above zero the error is that of the part
below: 7e-7 at most, and less than 8e-6 of the value."""
import numpy as np
import pytest
import torch
from scipy.special import ndtr

import paper_2105_14450_amd as c3

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,residual", [(4, 8192, False), (256, 1024, False), (4096, 1024, False), (256, 1024, True)])
def test_gelu_value_by_value(M, K, residual):
    """Few rows, the ring and the tuned kernel; rows in whole runs, with and without a residual (of zeros)."""
    N = 8192
    small = np.concatenate([[0.0], 2.0 ** -np.arange(1.0, 100.0, 3.0)])
    z = np.concatenate([np.linspace(-12.0, 12.0, N - 2 * small.size), small, -small]).astype(np.float32)
    d = c3.make_desc(1, M, K, N, in_dtype=c3.BF16, shard_dtype=c3.BF16)
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    Y, bias = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.from_numpy(z).cuda()
    e = c3.make_epilogue(c3.ACT_GELU, bias=bias, residual=zeros(M, N) if residual else None, residual_dtype=c3.BF16)
    nb = c3.cube3d_epilogue_workspace_bytes(d, c3.OP_FWD)
    c3.virtual_cube_linear_fwd_fused(d, e, zeros(M, K), zeros(K, N), Y, torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None)
    torch.cuda.synchronize()
    assert torch.equal(Y, Y[:1].expand(M, N))
    got, zd = Y[0].double().cpu().numpy(), z.astype(np.float64)
    want = zd * ndtr(zd)
    limit = 2.0 ** -8 * 1.001 * np.abs(want) + np.where(np.abs(zd) <= 6.0, 8e-6 * np.abs(want), 5e-14)
    bad = ~(np.abs(got - want) <= limit)
    assert not bad.any(), "worst at z = %g" % zd[np.argmax(np.abs(got - want) / np.maximum(limit, 1e-300))]
