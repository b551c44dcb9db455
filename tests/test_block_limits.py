"""Host side of the operators around the linear layers at sizes that no memory holds: a status, never the end of the process (no GPU)."""
import ctypes
import os

import pytest
import torch

import paper_2105_14450_amd as c3
from paper_2105_14450_amd import binding as b

SIZES = [1, 1600, 1 << 20, (1 << 31) - 1600, 1 << 31, 1 << 36, 1 << 44, 1 << 47, 1 << 55, 1 << 62, (1 << 63) - 1]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2105_14450_amd import build
        build.build()
    return b.load()


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would run")
@pytest.mark.parametrize("q", [1, 40])
def test_sizes_that_no_memory_holds(lib, q):
    at = lambda k: (1 << 40) + (k << 58)      # far from each other
    everything = ctypes.c_size_t(-1).value
    for M in SIZES:
        for N in SIZES:
            M, N = M // (q * q) * q * q, N // (q * q) * q * q
            if M < 1 or N < 1:
                continue
            d = c3.make_desc(q, M, q * 64, N, in_dtype=c3.BF16, shard_dtype=c3.BF16)
            large = M * N > 1 << 44
            nb = lib.cube3d_epilogue_workspace_bytes(ctypes.byref(d), c3.OP_BIAS_BWD)
            assert (nb == 0) == large and nb < 1 << 47
            rc = lib.virtual_cube_linear_epilogue_bwd(ctypes.byref(d), c3.ACT_GELU, c3.BF16, c3.BF16, c3.BF16, at(0), at(1), at(2), at(3), at(4),
                                                      everything, None)
            # (more columns than one launch takes are refused below 2^44 elements too)
            assert rc == c3.ESHAPE if large else rc in (c3.ESHAPE, c3.ELAUNCH)
            lib.cube3d_epilogue_workspace_bytes(ctypes.byref(d), c3.OP_FWD)
            e = b.Epilogue(c3.ACT_GELU, c3.BF16, c3.BF16, at(5), at(6), at(7))
            rc = lib.virtual_cube_linear_fwd_fused(ctypes.byref(d), ctypes.byref(e), at(0), at(1), at(2), at(3), everything, None)
            # (matrices too long for the distances between these addresses overlap)
            assert rc == c3.ESHAPE if max(M, N) >= 1 << 31 else rc in (c3.ESHAPE, c3.ELAUNCH) + (c3.EINVAL,) * large
            m, nd, p = c3.make_matrix(q, M, N, 0, 2, 0, c3.BF16), c3.make_norm(pre=2, post=1), b.NormParams()
            fits = M < 1 << 31 and N <= (1 << 31) - (1 << 16)
            assert (lib.cube3d_norm_workspace_bytes(ctypes.byref(m), ctypes.byref(nd)) > 0) == fits
            rc = lib.virtual_cube_norm_bwd(ctypes.byref(m), ctypes.byref(nd), ctypes.byref(p), *[at(k) for k in range(7)], ctypes.byref(p), at(7),
                                           everything, None)
            assert rc in ((c3.ELAUNCH,) + (c3.EINVAL,) * large if fits else (c3.ESHAPE,))
