"""What the binding refuses by itself ahead of the operators around the linear layers (no GPU: stand-ins for device tensors)."""
import pytest

import paper_2105_14450_amd as c3
from paper_2105_14450_amd import binding as b


class Stand:
    """As much of a device tensor as the binding looks at; never dereferenced: every call ends before the library."""
    is_cuda = True

    def __init__(self, n=64, size=4, device=0):
        self.n, self.size, self.device = n, size, device

    def numel(self):
        return self.n

    def element_size(self):
        return self.size

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x100000


class Stream:
    cuda_stream = 0

    def __init__(self, device):
        self.device_index = device


@pytest.fixture
def two_devices(monkeypatch):
    monkeypatch.setattr(b, "_one_device", False)
    monkeypatch.setattr(b, "_current_device", lambda: 0)

    def launched():
        raise AssertionError("the call went on to the library")
    monkeypatch.setattr(b, "load", launched)


def test_tensor_lists_count_elements_of_their_type():
    for size, n, code, elements in ((1, 64, c3.F32, 16), (1, 64, c3.BF16, 32), (2, 64, c3.BF16, 64), (4, 64, c3.F32, 64), (4, 0, c3.F32, 0)):
        t = c3.make_tensor_list([Stand(n, size)], [code])
        assert t.array[0].n == elements and bool(t.array[0].data) == (n > 0)
    for size, n, code in ((1, 63, c3.F32), (2, 33, c3.F32), (1, 5, c3.BF16), (4, 4, 9)):
        with pytest.raises(ValueError):
            c3.make_tensor_list([Stand(n, size)], [code])
    with pytest.raises(ValueError):
        c3.make_tensor_list([Stand()], [c3.F32, c3.F32])


def test_tensors_of_another_device(two_devices):
    here, away = Stand(), Stand(device=1)
    desc = c3.make_desc(1, 64, 64, 64)
    m, norm = c3.make_matrix(1, 64, 64, 0, 2, 0, c3.BF16), c3.make_norm(pre=c3.NORM_RMS)

    def refused(call):
        with pytest.raises(ValueError, match="device"):
            call()

    def each(call, n):
        for k in range(n):
            refused(lambda: call(*[away if i == k else here for i in range(n)]))
    each(lambda x, w, y, ws: c3.virtual_cube_linear_fwd_fused(desc, c3.make_epilogue(), x, w, y, ws), 4)
    each(lambda bias, r, z: c3.virtual_cube_linear_fwd_fused(desc, c3.make_epilogue(bias=bias, residual=r, z=z), here, here, here), 3)
    each(lambda *t: c3.virtual_cube_linear_epilogue_bwd(desc, c3.ACT_GELU, c3.BF16, c3.BF16, c3.BF16, *t), 5)
    none = c3.make_norm_params()
    each(lambda *t: c3.virtual_cube_norm_fwd(m, norm, none, *t), 5)
    each(lambda *p: c3.virtual_cube_norm_fwd(m, norm, c3.make_norm_params(*p), here, here, here, here), 5)
    each(lambda st, dr, dn, r, u, dx, du, ws: c3.virtual_cube_norm_bwd(m, norm, none, st, dr, dn, r, u, dx, du, none, ws), 8)
    each(lambda *p: c3.virtual_cube_norm_bwd(m, norm, none, *[here] * 7, c3.make_norm_params(*p), here), 5)
    each(lambda *p: c3.virtual_cube_norm_bwd(m, norm, c3.make_norm_params(*p), *[here] * 7, none, here), 5)
    lists = lambda *t: c3.make_tensor_list(t, [c3.F32] * len(t))
    double = Stand(1, 8)
    each(lambda g, norm, ws: c3.cube3d_grad_norm(lists(here, g), double, norm, ws), 3)
    each(lambda g, o: c3.cube3d_grad_clip(lists(here, g), lists(here, o), double, 1.0), 2)
    refused(lambda: c3.cube3d_grad_norm(lists(here), Stand(1, 8, device=1)))
    refused(lambda: c3.cube3d_grad_clip(lists(here), lists(here), Stand(1, 8, device=1), 1.0))
    refused(lambda: c3.cube3d_grad_clip(lists(here), lists(here), double, 1.0, stream=Stream(1)))
    refused(lambda: c3.virtual_cube_norm_fwd(m, norm, none, here, None, None, here, stream=Stream(1)))
    # where everything is in one place, or empty, the call goes on
    for call in (lambda: c3.cube3d_grad_clip(lists(here, Stand(0, 4, device=-1)), lists(here, Stand(0, 4, device=-1)), double, 1.0, stream=Stream(0)),
                 lambda: c3.virtual_cube_linear_fwd_fused(desc, b.Epilogue(c3.ACT_NONE), here, here, here)):
        with pytest.raises(AssertionError, match="library"):
            call()


def test_types_of_the_sums(two_devices):
    t = c3.make_tensor_list([Stand()], [c3.F32])
    for bad in (dict(sumsq=Stand(1, 4)), dict(sumsq=Stand(0, 8)), dict(sumsq=Stand(1, 8), norm=Stand(1, 8)), dict(sumsq=Stand(1, 8), norm=Stand(1, 2))):
        with pytest.raises(ValueError, match="float"):
            c3.cube3d_grad_norm(t, **bad)
    with pytest.raises(ValueError, match="float64"):
        c3.cube3d_grad_clip(t, t, Stand(1, 4), 1.0)
    with pytest.raises(ValueError, match="as many"):
        c3.cube3d_grad_clip(t, c3.make_tensor_list([], []), Stand(1, 8), 1.0)
