"""The norms' backward pass on rows of 8193 to 16384 columns, several rows a workgroup, with one and with both norms and as many
vectors' gradients as leave the column sums in LDS; and with one more, which leaves them to the passes for any size."""
import pytest

from tests.test_gpu_norm import NAMES, Problem, check_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q,axis,rows,cols,most", [(1, "y", 700, 9216, 4), (2, "z", 600, 8256, 4), (1, "z", 530, 12296, 2), (1, "y", 600, 11520, 3),
                                                   (1, "y", 520, 16384, 2)])
@pytest.mark.parametrize("post,pre,stream", [("layer", "rms", "f32"), ("rms", "layer", "bf16"), ("layer", "none", "bf16"), ("none", "layer", "f32")])
def test_several_rows_a_workgroup(q, axis, rows, cols, most, post, pre, stream):
    pr = Problem(q, axis, rows, cols, stream, "bf16", post, pre)
    possible = [k for k in NAMES if k == "gate" or (post if k.startswith("post") else pre) != "none"]
    # 256 workgroups take two to three rows each
    check_backward(pr, wanted=possible[:most])
    check_backward(pr, wanted=possible[-most:], in_place=True)
    if len(possible) > most:
        check_backward(pr, wanted=possible[:most + 1])
