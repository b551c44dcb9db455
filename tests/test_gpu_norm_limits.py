"""The norms' backward pass on rows of more columns than a grid dimension has room for.  Integers: exact."""
import pytest
import torch

import paper_2105_14450_amd as c3

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [(1 << 28) + 8, (1 << 30) + 1])
def test_columns_past_one_launch(cols):
    """2^28 columns and more: 2^22 workgroups of 1024 lanes write a vector's gradient; 2^30 single ones: 2^24 workgroups of 256 lanes
    form its partial sums.  One row, a gate and a scale, no norm: dg = s dr u, du = s dr."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    draw = lambda: torch.randint(-4, 5, (cols,), device="cuda", generator=gen, dtype=torch.int8).to(torch.bfloat16)
    dr, u = draw(), draw()
    du, dgate = torch.full_like(dr, float("nan")), torch.full((cols,), float("nan"), device="cuda")
    m = c3.make_matrix(1, 1, cols, c3.AXIS_X, c3.AXIS_Z, c3.SPLIT_ROWS, c3.BF16)
    norm = c3.make_norm(scale=0.5)
    ws = torch.empty(c3.cube3d_norm_workspace_bytes(m, norm), dtype=torch.uint8, device="cuda")
    c3.virtual_cube_norm_bwd(m, norm, c3.make_norm_params(), None, dr, None, None, u, None, du, c3.make_norm_params(gate=dgate), ws)
    torch.cuda.synchronize()
    for at in range(0, cols, 1 << 27):
        part = slice(at, at + (1 << 27))
        assert torch.equal(du[part], dr[part] * 0.5)
        assert torch.equal(dgate[part], dr[part].float() * u[part].float() * 0.5)
