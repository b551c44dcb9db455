"""The operators around the linear layers on arrays of more than 2^31 elements: offsets past 32 bits.  Integers where the result is exact;
else the rounding of the stored type (2^-8 of the value) and 2e-5 of the terms' size for the fp32 evaluation (sums of 8200
terms: at most 8200 / 64 + 24 additions on the way of any, 153 x 2^-24 = 1e-5)."""
import pytest
import torch

import paper_2105_14450_amd as c3

pytestmark = pytest.mark.gpu

ROWS, COLS = 262200, 8200


def some_rows(rows):
    return torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")


def integers(shape, seed, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-4, 5, shape, device="cuda", generator=gen, dtype=torch.int8).to(dtype)


def normal(shape, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def near(got, want, size):
    assert bool(((got.double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 2e-5 * size).all())


def test_norm():
    assert ROWS * COLS > 1 << 31
    x, dn, dr = (normal((1, ROWS, COLS), s) for s in (1, 2, 3))
    gamma = normal((1, COLS), 4).float()
    n, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((ROWS, 4), device="cuda")
    dgamma = torch.empty_like(gamma)
    m, norm = c3.make_matrix(1, ROWS, COLS, c3.AXIS_X, c3.AXIS_Z, c3.SPLIT_ROWS, c3.BF16), c3.make_norm(pre=c3.NORM_RMS)
    p = c3.make_norm_params(pre_gamma=gamma)
    c3.virtual_cube_norm_fwd(m, norm, p, x, None, None, n, stats)
    ws = torch.empty(c3.cube3d_norm_workspace_bytes(m, norm), dtype=torch.uint8, device="cuda")
    c3.virtual_cube_norm_bwd(m, norm, p, stats, dr, dn, x, None, dx, None, c3.make_norm_params(pre_gamma=dgamma), ws)
    torch.cuda.synchronize()
    rows = some_rows(ROWS)
    v, t, add, g = x[0, rows].double(), dn[0, rows].double(), dr[0, rows].double(), gamma[0].double()
    rstd = 1.0 / ((v * v).mean(1, keepdim=True) + 1e-5).sqrt()
    near(n[0, rows], v * rstd * g, (v * rstd * g).abs())
    hat, tg = v * rstd, t * g
    near(dx[0, rows], add + rstd * (tg - hat * (tg * hat).mean(1, keepdim=True)),
         add.abs() + rstd * (tg.abs() + hat.abs() * (tg * hat).abs().mean(1, keepdim=True)))
    want, size = torch.zeros(COLS, dtype=torch.float64, device="cuda"), torch.zeros(COLS, dtype=torch.float64, device="cuda")
    for lo in range(0, ROWS, 8192):
        a = x[0, lo:lo + 8192].double()
        a = a / ((a * a).mean(1, keepdim=True) + 1e-5).sqrt() * dn[0, lo:lo + 8192].double()
        want += a.sum(0)
        size += a.abs().sum(0)
    # a lane adds at most 1100 rows, then come 256 groups in 16 runs; a term's own error is 16 of such steps
    assert bool(((dgamma[0].double() - want).abs() <= (1100 + 32 + 16) * 2.0 ** -24 * size).all())


def test_epilogue_bwd():
    z, dy = integers((1, ROWS, COLS), 5), integers((1, ROWS, COLS), 6)
    dz, db = torch.empty_like(z), torch.empty((1, COLS), device="cuda")
    d = c3.make_desc(1, ROWS, 1, COLS, in_dtype=c3.BF16, shard_dtype=c3.BF16)
    ws = torch.empty(c3.cube3d_epilogue_workspace_bytes(d, c3.OP_BIAS_BWD), dtype=torch.uint8, device="cuda")
    c3.virtual_cube_linear_epilogue_bwd(d, c3.ACT_RELU, c3.BF16, c3.BF16, c3.BF16, z, dy, dz, db, ws)
    want = torch.zeros(COLS, dtype=torch.int64, device="cuda")
    for lo in range(0, ROWS, 8192):
        part = torch.where(z[0, lo:lo + 8192] > 0, dy[0, lo:lo + 8192], torch.zeros_like(dy[0, :1]))
        assert torch.equal(dz[0, lo:lo + 8192], part)
        want += part.long().sum(0)
    assert torch.equal(db[0].long(), want)      # sums below 2^24


@pytest.mark.parametrize("K,N", [(16, 32800), (256, 32800), (256, 32801)])
def test_linear(K, N):
    M = 65600
    assert M * N > 1 << 31
    X, W, R = integers((1, M, K), 7), integers((1, K, N), 8), integers((1, M, N), 9)
    b = integers((1, N), 10, torch.float32)
    Y, Z = torch.empty_like(R), torch.empty((1, M, N), device="cuda")
    d = c3.make_desc(1, M, K, N, in_dtype=c3.BF16, shard_dtype=c3.BF16)
    for residual, z in ((R, None), (None, Z), (R, Z)):
        Y.fill_(float("nan"))
        c3.virtual_cube_linear_fwd_fused(d, c3.make_epilogue(c3.ACT_RELU, bias=b, residual=residual, z=z, z_dtype=c3.F32), X, W, Y)
        rows = some_rows(M)
        want = (X[0, rows].float().cpu().double() @ W[0].float().cpu().double() + b[0].cpu().double()).cuda()
        if z is not None:
            assert torch.equal(z[0, rows].double(), want)
        want = want.clamp_min(0) + (0 if residual is None else R[0, rows].double())
        assert torch.equal(Y[0, rows], want.to(torch.bfloat16))
        assert not bool(torch.isnan(Y).any())
