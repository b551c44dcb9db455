"""Host-side refusals of results and workspaces that overlap something else of the call (no GPU: nothing is launched).  The calls that
are not refused end as a launch without a device does."""
import ctypes
import os

import pytest
import torch

import paper_2105_14450_amd as c3
from paper_2105_14450_amd import binding as b

STEP = 0x1000000
A = 0x10000000
at = lambda k: A + STEP * k


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2105_14450_amd import build
        build.build()
    return b.load()


def refused(call, arrays, result, other, sizes, in_place=False):
    """Every way for `result` to lie on `other`: its first and last 16 bytes, inside, around; and not right behind or ahead of it."""
    base, ro, rs = arrays[other], sizes[other], sizes[result]
    for where in (base + 16, base + ro - 16, base - rs + 16, base - 16):
        assert call(**{**arrays, result: where}) == c3.EINVAL, (result, other, where - base)
    assert (call(**{**arrays, result: base}) == c3.EINVAL) != in_place, (result, other)


def allowed(status):
    return status not in (c3.EINVAL, c3.ESHAPE, c3.EDTYPE, c3.EWORKSPACE)


# without a device the library ends with a launch error; on a machine with one the addresses below may not be touched
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would run")


def fused(lib, M, K, N, q=1, y_type=c3.BF16, r_type=c3.BF16, z_type=c3.F32):
    d = c3.make_desc(q, M, K, N, in_dtype=c3.BF16, shard_dtype=y_type)
    need = lib.cube3d_epilogue_workspace_bytes(ctypes.byref(d), c3.OP_FWD)
    size = {c3.BF16: 2, c3.F32: 4}
    sizes = {"x": M * K * 2, "w": K * N * 2, "bias": q * N * 4, "r": M * N * size[r_type], "z": M * N * size[z_type], "y": M * N * size[y_type], "ws": need}
    arrays = {k: at(8 * i) for i, k in enumerate(sizes)}

    def call(x, w, bias, r, z, y, ws):
        e = b.Epilogue(c3.ACT_GELU, r_type, z_type, bias, r, z)
        return lib.virtual_cube_linear_fwd_fused(ctypes.byref(d), ctypes.byref(e), x, w, y, ws if need else None, need, None)
    return call, arrays, sizes


@no_device
@pytest.mark.parametrize("M,K,N,q", [(4, 8192, 512, 1), (256, 1024, 512, 1), (64, 1024, 512, 2), (130, 336, 72, 1)])
def test_linear_fwd_fused(lib, M, K, N, q):
    call, arrays, sizes = fused(lib, M, K, N, q)
    assert allowed(call(**arrays))
    for other in ("x", "w", "bias", "z", "r"):
        refused(call, arrays, "y", other, sizes, in_place=other == "r")
    for other in ("x", "w", "bias", "r", "y"):
        refused(call, arrays, "z", other, sizes)
    if sizes["ws"]:
        for other in ("x", "w", "bias", "r", "z", "y"):
            refused(call, arrays, "ws", other, sizes)
    # side by side
    assert allowed(call(**{**arrays, "y": arrays["x"] + sizes["x"]})) and allowed(call(**{**arrays, "z": arrays["y"] + sizes["y"]}))
    # operands may share memory
    assert allowed(call(**{**arrays, "r": arrays["x"], "bias": arrays["w"]}))
    call, arrays, sizes = fused(lib, M, K, N, q, y_type=c3.F32)
    refused(call, arrays, "y", "r", sizes)


@no_device
@pytest.mark.parametrize("M,N,q", [(256, 512, 2), (130, 77, 1)])
def test_linear_epilogue_bwd(lib, M, N, q):
    d = c3.make_desc(q, M, q, N)
    need = lib.cube3d_epilogue_workspace_bytes(ctypes.byref(d), c3.OP_BIAS_BWD)
    sizes = {"z": M * N * 4, "dy": M * N * 2, "dz": M * N * 2, "db": q * N * 4, "ws": need}
    sizes = {k: v // 16 * 16 for k, v in sizes.items()}     # (addresses are multiples of 16)
    arrays = {k: at(i) for i, k in enumerate(sizes)}

    def call(z, dy, dz, db, ws):
        return lib.virtual_cube_linear_epilogue_bwd(ctypes.byref(d), c3.ACT_GELU, c3.F32, c3.BF16, c3.BF16, z, dy, dz, db, ws, need, None)
    assert allowed(call(**arrays))
    refused(call, arrays, "dz", "z", sizes)
    refused(call, arrays, "dz", "dy", sizes, in_place=True)
    refused(call, arrays, "db", "dz", sizes)
    for other in ("z", "dy", "dz", "db"):
        refused(call, arrays, "ws", other, sizes)
    assert allowed(call(**{**arrays, "db": arrays["dy"]}))      # (written behind everything that is read)
    assert allowed(call(**{**arrays, "db": None, "ws": arrays["z"]}))


NAMES = ("post_gamma", "post_beta", "gate", "pre_gamma", "pre_beta")


def norms(q, rows, cols, stream):
    m = c3.make_matrix(q, rows, cols, c3.AXIS_X, c3.AXIS_Z, c3.SPLIT_ROWS, stream)
    return m, c3.make_norm(pre=c3.NORM_LAYER, post=c3.NORM_LAYER, block_dtype=c3.BF16), rows * cols * (4 if stream == c3.F32 else 2), rows * cols * 2


@no_device
@pytest.mark.parametrize("q,rows,cols,stream", [(2, 64, 512, c3.BF16), (1, 96, 128, c3.F32)])
def test_norm_fwd(lib, q, rows, cols, stream):
    m, nd, se, be = norms(q, rows, cols, stream)
    sizes = {"x": se, "u": be, "r": se, "n": be, "stats": rows * 16, **{k: q * cols * 4 for k in NAMES}}
    arrays = {k: at(i) for i, k in enumerate(sizes)}

    def call(x, u, r, n, stats, **p):
        return lib.virtual_cube_norm_fwd(ctypes.byref(m), ctypes.byref(nd), ctypes.byref(b.NormParams(**p)), x, u, r, n, stats, None)
    assert allowed(call(**arrays))
    for result, others in (("r", ("x", "u", "n", "stats") + NAMES), ("n", ("x", "u", "r", "stats") + NAMES), ("stats", ("x", "u", "r", "n") + NAMES)):
        for other in others:
            refused(call, arrays, result, other, sizes, in_place=(result, other) == ("r", "x"))
    assert allowed(call(**{**arrays, "u": arrays["x"], "gate": arrays["pre_gamma"]}))
    # what is ignored may lie anywhere
    nd.pre_kind = c3.NORM_NONE
    assert allowed(call(**{**arrays, "n": None, "pre_beta": arrays["r"]}))


@no_device
@pytest.mark.parametrize("q,rows,cols,stream", [(2, 64, 512, c3.BF16), (1, 96, 128, c3.F32)])
def test_norm_bwd(lib, q, rows, cols, stream):
    m, nd, se, be = norms(q, rows, cols, stream)
    need = lib.cube3d_norm_workspace_bytes(ctypes.byref(m), ctypes.byref(nd))
    sizes = {"stats": rows * 16, "dr": se, "dn": be, "r": se, "u": be, "dx": se, "du": be, "ws": need, **{k: q * cols * 4 for k in NAMES},
             **{"d_" + k: q * cols * 4 for k in NAMES}}
    arrays = {k: at(i) for i, k in enumerate(sizes)}

    def call(stats, dr, dn, r, u, dx, du, ws, **p):
        params, grads = (b.NormParams(**{k: p[pre + k] for k in NAMES}) for pre in ("", "d_"))
        return lib.virtual_cube_norm_bwd(ctypes.byref(m), ctypes.byref(nd), ctypes.byref(params), stats, dr, dn, r, u, dx, du, ctypes.byref(grads), ws,
                                         need, None)
    assert allowed(call(**arrays))
    read = ("stats", "dr", "dn", "r", "u") + NAMES
    grads = tuple("d_" + k for k in NAMES)
    for result, others in (("dx", read + ("du",) + grads), ("du", read + ("dx",) + grads), ("ws", read + ("dx", "du") + grads), ("d_gate", ("dx", "du", "ws", "d_pre_beta"))):
        for other in others:
            refused(call, arrays, result, other, sizes, in_place=(result, other) == ("dx", "dr"))
    assert allowed(call(**{**arrays, "d_gate": arrays["gate"], "d_pre_beta": arrays["dn"]}))      # (written behind everything that is read)


@no_device
def test_gradients(lib):
    grads = (b.Tensor * 2)(b.Tensor(at(0), 1000, c3.F32), b.Tensor(at(1), 5000, c3.BF16))
    out = (b.Tensor * 2)(b.Tensor(at(2), 1000, c3.BF16), b.Tensor(at(3), 5000, c3.F32))
    need = lib.cube3d_grad_norm_workspace_bytes(grads, 2)
    norm = lambda sumsq=at(4), norm=at(5), ws=at(6): lib.cube3d_grad_norm(grads, 2, 1.0, sumsq, norm, ws, need, None)
    clip = lambda sumsq: lib.cube3d_grad_clip(grads, out, 2, 1.0, 1.0, sumsq, None)
    assert allowed(norm()) and allowed(clip(at(4)))
    assert norm(norm=at(4)) == c3.EINVAL and norm(norm=at(4) + 4) == c3.EINVAL and allowed(norm(norm=at(4) + 8)) and allowed(norm(norm=at(4) - 4))
    for ws in (at(0), at(0) + 3984, at(0) - need + 16 if need > 16 else at(0), at(1) + 9984):
        assert norm(ws=ws) == c3.EINVAL
    assert allowed(norm(ws=at(0) + 4000)) and allowed(norm(ws=at(1) + 10000))
    for sumsq in (at(2), at(2) + 1992, at(3) + 19992):
        assert clip(sumsq) == c3.EINVAL
    assert allowed(clip(at(2) + 2000)) and allowed(clip(at(2) - 8))
