"""Gradient norms at the end of fp32's range: what the stored norm says is what clipping does."""
import numpy as np
import pytest
import torch

import paper_2105_14450_amd as c3

pytestmark = pytest.mark.gpu


def clip(grads, max_norm, scale):
    lst = c3.make_tensor_list(grads)
    sumsq, norm = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(c3.cube3d_grad_norm_workspace_bytes(lst), dtype=torch.uint8, device="cuda")
    c3.cube3d_grad_norm(lst, sumsq, norm, ws, scale=scale)
    out = [torch.full(g.shape, float("nan"), device="cuda") for g in grads]
    c3.cube3d_grad_clip(lst, c3.make_tensor_list(out), sumsq, max_norm, scale=scale)
    torch.cuda.synchronize()
    return norm.item(), out


@pytest.mark.parametrize("n,scale", [(4, 1.0), (4, 0.5), (1, 1.0), (9000, 1.0), (9000, 2.0 ** -7), (2, 0.75)])
def test_a_norm_past_fp32(n, scale):
    """n elements of +-2^127 beside small ones: the norm is 2^127 sqrt(n), and past fp32's largest value for n >= 4."""
    g = torch.full((n,), 2.0 ** 127, device="cuda")
    g[::2] *= -1.0
    small = torch.tensor([3.0, -5.0], device="cuda", dtype=torch.bfloat16)
    want, top = scale * 2.0 ** 127 * np.sqrt(n), float(np.finfo(np.float32).max)
    norm, (a, b) = clip([g, small], 2.0 ** 100, scale)
    if want > top * (1 + 2.0 ** -25):
        assert norm == float("inf")
        f, steps = scale, 0.0                # powers of two and small integers: exact
    else:
        assert abs(norm - want) <= 2.0 ** -24 * 1.001 * want
        f, steps = scale * 2.0 ** 100 / want, 2.001 * 2.0 ** -24     # the factor's rounding and the product's
    for got, have in ((a, g), (b, small)):
        ref = have.double() * f
        assert bool(((got.double() - ref).abs() <= steps * ref.abs()).all())
