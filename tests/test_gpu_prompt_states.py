"""`prompt_attn` on values of very different sizes: channels far below their row's largest, with tokens in parts as they are.
Reference and tolerances are those of tests/test_gpu_prompt_attn.py: they go by a channel's own terms."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_prompt_attn import PAGE, Problem  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, PAGE])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("ratio", [16, 24, 60])
def test_channels_far_below_their_row_s_largest(dtype, page, d, ratio):
    for new, past in (([1, 3], [1500, 700]), ([90], [2000]), ([300, 200], [0, 0])):
        p = Problem(dtype, 4, 2, d, new, past, page=page, seed=d + ratio)
        p.v[..., 0] *= 2.0 ** ratio
        p.v[..., 3] *= 2.0 ** (ratio // 2)
        p.check()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_parts_whose_rows_differ_in_size(d):
    """A late stretch of tokens with values 2^40 times the rest, seen by the last rows only."""
    p = Problem("bf16", 4, 1, d, [60], [1700], seed=d)
    p.v[1720:] *= 2.0 ** 40
    p.check()
