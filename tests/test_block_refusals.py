"""Host-side refusals of the operators around the linear layers: every bad call ends before anything is launched (no GPU)."""
import ctypes
import os

import pytest

import paper_2105_14450_amd as c3
from paper_2105_14450_amd import binding as b

A = 0x100000      # an aligned address per argument, never dereferenced: validation fails first
X, W, Y, R, Z, U, N, D, E, WS = (A + 0x100000 * k for k in range(10))
ODD = A + 8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2105_14450_amd import build
        build.build()
    return b.load()


def desc(**kw):
    args = dict(q=2, M=256, K=128, N=128, in_dtype=c3.BF16, shard_dtype=c3.BF16)
    args.update(kw)
    return c3.make_desc(**args)


def test_mirrors_match_the_header():
    assert ctypes.sizeof(b.Epilogue) == 40 and b.Epilogue.bias_diag.offset == 16
    assert ctypes.sizeof(b.Norm) == 24 and b.Norm.post_eps.offset == 12
    assert ctypes.sizeof(b.NormParams) == 40 and b.NormParams.pre_beta.offset == 32
    assert ctypes.sizeof(b.Tensor) == 24 and b.Tensor.dtype.offset == 16


def fused(lib, d=None, act=c3.ACT_GELU, bias=None, residual=None, residual_dtype=c3.BF16, z=None, z_dtype=c3.BF16, x=X, w=W, y=Y,
          ws=WS, ws_bytes=1 << 40, epilogue=True):
    e = b.Epilogue(act, residual_dtype, z_dtype, bias, residual, z)
    d = desc() if d is None else d
    return lib.virtual_cube_linear_fwd_fused(ctypes.byref(d), ctypes.byref(e) if epilogue else None, x, w, y, ws, ws_bytes, None)


def test_linear_fwd_fused(lib):
    assert lib.virtual_cube_linear_fwd_fused(None, None, X, W, Y, WS, 1 << 40, None) == c3.EINVAL
    assert fused(lib, epilogue=False) == c3.EINVAL
    for act in (-1, 3, 99):
        assert fused(lib, act=act) == c3.EINVAL
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(x=ODD), dict(w=ODD), dict(y=ODD), dict(bias=ODD), dict(residual=ODD),
                dict(z=ODD), dict(ws=ODD), dict(z=Y), dict(z=R, residual=R), dict(residual=Y, residual_dtype=c3.F32)):
        assert fused(lib, **bad) == c3.EINVAL, bad
    for bad in (dict(residual=R, residual_dtype=c3.FP8_E4M3), dict(residual=R, residual_dtype=7), dict(z=Z, z_dtype=c3.FP8_E4M3)):
        assert fused(lib, **bad) == c3.EDTYPE, bad
    for bad in (dict(M=258), dict(K=127), dict(N=130), dict(M=0), dict(M=1 << 33)):
        assert fused(lib, desc(**bad)) == c3.ESHAPE, bad
    assert fused(lib, desc(q=0)) == c3.EINVAL
    assert fused(lib, desc(in_axis=c3.AXIS_X)) == c3.EINVAL
    assert fused(lib, desc(in_dtype=5)) == c3.EDTYPE
    assert fused(lib, desc(shard_dtype=c3.FP8_E4M3)) == c3.EDTYPE
    assert fused(lib, desc(in_dtype=c3.FP8_E4M3, scale_w=0.0)) == c3.EINVAL
    assert lib.cube3d_epilogue_workspace_bytes(None, c3.OP_FWD) == 0
    assert lib.cube3d_epilogue_workspace_bytes(ctypes.byref(desc(M=258)), c3.OP_BIAS_BWD) == 0
    assert lib.cube3d_epilogue_workspace_bytes(ctypes.byref(desc()), c3.OP_BWD_DX) == 0


def test_no_activation_is_not_an_elementwise_call(lib):
    assert lib.cube3d_activation_fwd(c3.ACT_NONE, c3.F32, c3.F32, 64, X, Y, None) == c3.EINVAL


def test_linear_epilogue_bwd(lib):
    d = desc()
    need = lib.cube3d_epilogue_workspace_bytes(ctypes.byref(d), c3.OP_BIAS_BWD)
    assert need >= 128 * 4

    def call(kind=c3.ACT_GELU, zt=c3.BF16, gt=c3.BF16, dt=c3.BF16, z=Z, dy=Y, dz=D, db=E, ws=WS, ws_bytes=need, d=d):
        return lib.virtual_cube_linear_epilogue_bwd(ctypes.byref(d), kind, zt, gt, dt, z, dy, dz, db, ws, ws_bytes, None)
    for bad in (dict(kind=c3.ACT_NONE), dict(kind=-1), dict(z=None), dict(dy=None), dict(dz=None), dict(z=ODD), dict(dy=ODD), dict(dz=ODD),
                dict(db=ODD), dict(ws=ODD), dict(dz=Z), dict(dz=Y, dt=c3.F32), dict(d=desc(q=-1))):
        assert call(**bad) == c3.EINVAL, bad
    for bad in (dict(zt=c3.FP8_E4M3), dict(gt=c3.FP8_E4M3), dict(dt=c3.FP8_E4M3), dict(zt=9)):
        assert call(**bad) == c3.EDTYPE, bad
    assert call(ws=None) == c3.EWORKSPACE and call(ws_bytes=need - 1) == c3.EWORKSPACE
    assert call(d=desc(N=130)) == c3.ESHAPE


def matrix(rows=256, cols=128, q=2, row_axis=c3.AXIS_X, col_axis=c3.AXIS_Z, split=c3.SPLIT_ROWS, dtype=c3.BF16):
    return c3.make_matrix(q, rows, cols, row_axis, col_axis, split, dtype)


PARAMS = b.NormParams(*[A + 0x1000 * k for k in range(5)])
NOTHING = b.NormParams()


def test_norm_fwd(lib):
    def call(m=None, nd=None, params=PARAMS, x=X, u=U, r=R, n=N, stats=E):
        m = matrix() if m is None else m
        nd = c3.make_norm(pre=c3.NORM_LAYER, post=c3.NORM_RMS) if nd is None else nd
        return lib.virtual_cube_norm_fwd(ctypes.byref(m), ctypes.byref(nd), ctypes.byref(params) if params is not None else None, x, u, r, n,
                                         stats, None)
    assert lib.virtual_cube_norm_fwd(None, None, None, X, U, R, N, E, None) == c3.EINVAL
    assert lib.virtual_cube_norm_fwd(ctypes.byref(matrix()), None, ctypes.byref(PARAMS), X, U, R, N, E, None) == c3.EINVAL
    for bad in (dict(row_axis=c3.AXIS_Y), dict(split=c3.SPLIT_COLS), dict(col_axis=c3.AXIS_X), dict(q=0)):
        assert call(matrix(**bad)) == c3.EINVAL, bad
    for bad in (dict(rows=254), dict(cols=126), dict(cols=0), dict(q=1, rows=1 << 31), dict(q=1, cols=1 << 31)):
        assert call(matrix(**bad)) == c3.ESHAPE, bad
    assert call(matrix(dtype=c3.FP8_E4M3)) == c3.EDTYPE
    norm = lambda **kw: c3.make_norm(**{"pre": c3.NORM_LAYER, "post": c3.NORM_RMS, **kw})
    assert call(nd=norm(block_dtype=c3.FP8_E4M3)) == c3.EDTYPE
    nan, inf = float("nan"), float("inf")
    for bad in (dict(pre=3), dict(post=-1), dict(pre_eps=0.0), dict(post_eps=-1.0), dict(pre_eps=nan), dict(post_eps=inf), dict(scale=nan),
                dict(scale=inf), dict(scale=-inf)):
        assert call(nd=norm(**bad)) == c3.EINVAL, bad
    for bad in (dict(params=None), dict(x=None), dict(u=None), dict(r=None), dict(n=None), dict(x=ODD), dict(u=ODD), dict(r=ODD), dict(n=ODD),
                dict(stats=ODD), dict(n=X), dict(n=U), dict(n=R), dict(r=U), dict(params=b.NormParams(gate=ODD)),
                dict(u=None, r=None),                                                   # a norm behind a block that is not there
                dict(nd=norm(pre=c3.NORM_NONE)),                                        # n without a norm
                dict(nd=norm(pre=c3.NORM_NONE, post=c3.NORM_NONE), u=None, r=None, n=None)):
        assert call(**bad) == c3.EINVAL, bad


def test_norm_bwd(lib):
    nd0 = c3.make_norm(pre=c3.NORM_LAYER, post=c3.NORM_RMS)
    need = lib.cube3d_norm_workspace_bytes(ctypes.byref(matrix()), ctypes.byref(nd0))
    assert need > 0
    assert lib.cube3d_norm_workspace_bytes(None, ctypes.byref(nd0)) == 0
    assert lib.cube3d_norm_workspace_bytes(ctypes.byref(matrix(rows=254)), ctypes.byref(nd0)) == 0
    DR, DN, DX, DU = (A + 0x10000000 + 0x100000 * k for k in range(4))

    def call(m=None, nd=nd0, params=PARAMS, stats=E, dr=DR, dn=DN, r=R, u=U, dx=DX, du=DU, grads=PARAMS, ws=WS, ws_bytes=need):
        m = matrix() if m is None else m
        ref = lambda s: ctypes.byref(s) if s is not None else None
        return lib.virtual_cube_norm_bwd(ref(m), ref(nd), ref(params), stats, dr, dn, r, u, dx, du, ref(grads), ws, ws_bytes, None)
    none, pre, post = (c3.make_norm(pre=p, post=q) for p, q in ((0, 0), (c3.NORM_RMS, 0), (0, c3.NORM_RMS)))
    gate = b.NormParams(gate=A)
    for bad in (dict(params=None), dict(grads=None), dict(stats=None), dict(dn=None), dict(r=None), dict(u=None), dict(stats=ODD),
                dict(dr=ODD), dict(dn=ODD), dict(r=ODD), dict(u=ODD), dict(dx=ODD), dict(du=ODD), dict(ws=ODD),
                dict(dx=DN), dict(dx=R), dict(dx=U), dict(du=DN), dict(du=R), dict(du=U), dict(du=DR), dict(du=DX),
                dict(nd=pre), dict(nd=post), dict(nd=post, dn=None, grads=NOTHING, stats=None),
                dict(nd=pre, grads=gate, u=None, du=None), dict(nd=pre, grads=NOTHING, u=None),
                dict(nd=none, dn=None, dr=None, grads=NOTHING), dict(grads=NOTHING, dx=None, du=None),
                dict(grads=b.NormParams(pre_beta=ODD))):
        assert call(**bad) == c3.EINVAL, bad
    assert call(ws=None) == c3.EWORKSPACE and call(ws_bytes=need - 1) == c3.EWORKSPACE
    assert call(m=matrix(cols=126)) == c3.ESHAPE and call(m=matrix(dtype=c3.FP8_E4M3)) == c3.EDTYPE


def tensors(*items):
    return (b.Tensor * max(1, len(items)))(*[b.Tensor(*i) for i in items])


def test_gradients(lib):
    t = tensors((X, 100, c3.F32), (W, 50, c3.BF16))
    need = lib.cube3d_grad_norm_workspace_bytes(t, 2)
    assert need == 16
    big = tensors(*[(X, 1 << 30, c3.BF16)] * 300)
    assert 0 < lib.cube3d_grad_norm_workspace_bytes(big, 300) <= 3 * 256 * 8 * 8
    assert lib.cube3d_grad_norm_workspace_bytes(t, -1) == 0 and lib.cube3d_grad_norm_workspace_bytes(None, 2) == 0
    norm = lambda t=t, n=2, scale=1.0, s=R, out=Z, ws=WS, wb=need: lib.cube3d_grad_norm(t, n, scale, s, out, ws, wb, None)
    clip = lambda t=t, o=None, n=2, scale=1.0, mx=1.0, s=R: lib.cube3d_grad_clip(t, t if o is None else o, n, scale, mx, s, None)
    inf, nan = float("inf"), float("nan")
    for scale in (0.0, -1.0, inf, nan):
        assert norm(scale=scale) == c3.EINVAL and clip(scale=scale) == c3.EINVAL
    for mx in (0.0, -1.0, nan):
        assert clip(mx=mx) == c3.EINVAL
    assert norm(n=-1) == c3.EINVAL and norm(t=None) == c3.EINVAL and clip(n=-1) == c3.EINVAL
    assert norm(s=None) == c3.EINVAL and norm(s=R + 4) == c3.EINVAL and norm(out=Z + 2) == c3.EINVAL and norm(ws=ODD) == c3.EINVAL
    assert clip(s=None) == c3.EINVAL and clip(s=R + 4) == c3.EINVAL
    assert norm(ws=None) == c3.EWORKSPACE and norm(wb=need - 1) == c3.EWORKSPACE
    for bad, status in (((X, -1, c3.F32), c3.ESHAPE), ((X, 1 << 48, c3.F32), c3.ESHAPE), ((None, 5, c3.F32), c3.EINVAL),
                        ((ODD, 5, c3.F32), c3.EINVAL), ((X, 5, c3.FP8_E4M3), c3.EDTYPE), ((X, 5, 9), c3.EDTYPE)):
        t2 = tensors((W, 50, c3.BF16), bad)
        assert norm(t=t2) == status and clip(t=t2) == status and clip(o=t2) == status, bad
    assert clip(o=tensors((Y, 100, c3.F32), (Z, 51, c3.BF16))) == c3.ESHAPE


def test_results_of_clipping_may_not_overlap(lib):
    clip = lambda g, o: lib.cube3d_grad_clip(tensors(*g), tensors(*o), len(g), 1.0, 1.0, R, None)
    f, h = c3.F32, c3.BF16
    for g, o in (([(X, 64, f), (W, 64, f)], [(Y, 64, f), (Y, 64, f)]),                    # two results in one place
                 ([(X, 64, f), (X, 64, f)], [(X, 64, f), (X, 64, f)]),                    # the same array twice, in place
                 ([(X, 64, f)], [(X + 16, 64, f)]), ([(X + 16, 64, f)], [(X, 64, f)]),    # shifted
                 ([(X, 64, h)], [(X, 64, f)]), ([(X, 64, f)], [(X, 64, h)]),              # in place with another type
                 ([(X, 64, f), (W, 64, f)], [(W, 64, f), (X, 64, f)]),                    # swapped
                 ([(X, 64, f), (W, 64, f)], [(X, 64, f), (X + 128, 64, f)]),              # inside another one
                 ([(X, 4, f), (W, 64, f)], [(W + 240, 4, f), (Y, 64, f)])):               # on the end of another gradient
        assert clip(g, o) == c3.EINVAL, (g, o)


def test_norm_sizes_and_gradients_in_one_place(lib):
    nd = c3.make_norm(pre=c3.NORM_RMS)
    for cols, status in (((1 << 31) - 1, c3.ESHAPE), ((1 << 31) - (1 << 16) + 1, c3.ESHAPE), ((1 << 31) - (1 << 16), c3.EINVAL)):
        m = matrix(q=1, rows=1, cols=cols)      # (the last one is refused for its arguments)
        assert lib.virtual_cube_norm_fwd(ctypes.byref(m), ctypes.byref(nd), ctypes.byref(NOTHING), None, None, None, N, None, None) == status
    nd = c3.make_norm(pre=c3.NORM_LAYER, post=c3.NORM_LAYER)
    names = [f[0] for f in b.NormParams._fields_]
    for i, first in enumerate(names):
        for second in names[:i]:
            g = b.NormParams(**{first: A, second: A})
            assert lib.virtual_cube_norm_bwd(ctypes.byref(matrix()), ctypes.byref(nd), ctypes.byref(NOTHING), E, X, N, R, U, Y, D,
                                             ctypes.byref(g), WS, 1 << 40, None) == c3.EINVAL


def test_results_in_place_of_an_operand(lib):
    for bad in (dict(y=X), dict(y=W), dict(z=X), dict(z=W), dict(z=X, z_dtype=c3.F32)):
        assert fused(lib, **bad) == c3.EINVAL, bad
