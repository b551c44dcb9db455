"""NaN and infinities through the linear layer with activation and residual, on every kernel family and output stage: whatever
sizes, types and parts a call has, its answer is the same.  Integers elsewhere, so that every other element is compared bit for bit."""
import pytest
import torch

import paper_2105_14450_amd as c3

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8_e4m3": torch.float8_e4m3fn}
ACT = {"none": c3.ACT_NONE, "relu": c3.ACT_RELU, "gelu": c3.ACT_GELU}

# few rows in runs of the contraction, in one run, in blocks; ring tiles of 32, 64, 128 and more; tuned tiles of 256 and 128; loads of
# 4 bytes and of single elements; short contractions; rows of no whole pieces
SIZES = [(4, 8192, 512), (16, 4096, 2048), (128, 8192, 264), (20, 1024, 96), (256, 1024, 512), (1536, 2048, 1024), (2304, 512, 4096), (4096, 512, 4096),
         (1920, 512, 2176), (300, 516, 260), (130, 333, 77), (4096, 16, 1031), (512, 1024, 1004)]
# residual, Z, result: each output stage of its own and the general ones
PARTS = [(None, None, "bf16"), (None, "bf16", "bf16"), ("bf16", None, "bf16"), ("f32", None, "bf16"), ("bf16", "bf16", "bf16"), (None, "f32", "f32"),
         ("f32", None, "f32")]
ROW_NAN, ROW_INF = 1, 3


def operands(M, K, N, dtype):
    """Integers; a NaN in one row of X, and (where the type has them) an infinity in another whose sign the columns of W turn."""
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    draw = lambda shape, lo, hi: torch.randint(lo, hi, shape, device="cuda", generator=gen).float()
    X, W, R, b = draw((M, K), -4, 5), draw((K, N), -4, 5), draw((M, N), -4, 5), draw((N,), -4, 5)
    at = K // 2
    X[ROW_NAN, at] = float("nan")
    W[at] = torch.where(torch.arange(N, device="cuda") % 3 == 0, 1.0, -1.0)
    if dtype != "fp8_e4m3":
        X[ROW_INF, at] = float("inf")
    return X.to(TORCH[dtype]), W.to(TORCH[dtype]), R, b


def run(M, K, N, dtype, act, residual, z, out, X, W, R, b):
    d = c3.make_desc(1, M, K, N, in_dtype=c3.binding.DTYPE_CODES[dtype], shard_dtype=c3.binding.DTYPE_CODES[out])
    code = c3.binding.DTYPE_CODES
    Y = torch.full((M, N), 7.0, device="cuda", dtype=TORCH[out])
    Z = torch.full((M, N), 7.0, device="cuda", dtype=TORCH[z]) if z else None
    r = R.to(TORCH[residual]) if residual else None
    e = c3.make_epilogue(ACT[act], bias=b, residual=r, residual_dtype=code[residual or "f32"], z=Z, z_dtype=code[z or "f32"])
    nb = c3.cube3d_epilogue_workspace_bytes(d, c3.OP_FWD)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
    c3.virtual_cube_linear_fwd_fused(d, e, X, W, Y, ws)
    torch.cuda.synchronize()
    return Y, Z


def same(got, want):
    want = want.to(got.dtype)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], want[~nan])


def check_relu(M, K, N, dtype, parts):
    X, W, R, b = operands(M, K, N, dtype)
    ref = X.double() @ W.double() + b.double()
    assert bool(torch.isnan(ref[ROW_NAN]).all()) and int(torch.isnan(ref).any(1).sum()) == 1
    for residual, z, out in parts:
        Y, Z = run(M, K, N, dtype, "relu", residual, z, out, X, W, R, b)
        if z:
            same(Z, ref)
        same(Y, torch.where(ref <= 0, 0.0, ref) + (R.double() if residual else 0.0))


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp8_e4m3"])
def test_rectifier_keeps_nan(M, K, N, dtype):
    check_relu(M, K, N, dtype, PARTS)


@pytest.mark.parametrize("M,K,N", [(4, 2048, 256), (64, 4096, 520), (256, 512, 512), (1004, 1028, 1004), (130, 333, 77), (3001, 17, 1031)])
def test_rectifier_keeps_nan_in_fp32(M, K, N):
    check_relu(M, K, N, "f32", [p for p in PARTS if p[2] == "f32"] + PARTS[:1])


def check_gelu(M, K, N, dtype, parts):
    """Against z Phi(z) as it stands: +infinity stays, -infinity times zero is NaN, and NaN stays.  Finite ones: a bf16 rounding (2^-8) and
    1e-6, or 1e-6 and 4e-6 of the value in fp32 (the evaluation's own error; |z| is 1e4 at most, the sum exact)."""
    X, W, R, b = operands(M, K, N, dtype)
    ref = X.double() @ W.double() + b.double()
    if dtype != "fp8_e4m3":
        assert set(ref[ROW_INF].tolist()) == {float("inf"), -float("inf")}
    for residual, z, out in parts:
        Y, Z = run(M, K, N, dtype, "gelu", residual, z, out, X, W, R, b)
        if z:
            same(Z, ref)
        want = ref * torch.special.ndtr(ref) + (R.double() if residual else 0.0)
        if dtype != "fp8_e4m3":
            assert bool((want[ROW_INF].isnan() == (ref[ROW_INF] < 0)).all())
        fine = want.isfinite()
        assert torch.equal(Y.isnan(), want.isnan()) and torch.equal(Y[~fine & ~want.isnan()], want[~fine & ~want.isnan()].to(Y.dtype))
        size = want[fine].abs() + (R.double().abs()[fine] if residual else 0.0)
        assert bool(((Y[fine].double() - want[fine]).abs() <= (1.01 * 2.0 ** -8 if out == "bf16" else 4e-6) * size + 1e-6).all())


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp8_e4m3"])
def test_gelu_of_infinities_is_the_same_everywhere(M, K, N, dtype):
    check_gelu(M, K, N, dtype, PARTS)


@pytest.mark.parametrize("M,K,N", [(4, 2048, 256), (64, 4096, 520), (256, 512, 512), (1004, 1028, 1004), (130, 333, 77), (3001, 17, 1031)])
def test_gelu_of_infinities_in_fp32(M, K, N):
    check_gelu(M, K, N, "f32", [p for p in PARTS if p[2] == "f32"] + PARTS[:1])
