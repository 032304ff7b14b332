"""`accumulate_kv_weights`: head sizes between the padded ones, with rows enough for every kernel of both types."""
import pytest

from test_gpu_kv_weights import Problem

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 56, 88, 104, 136, 160, 184, 192, 200, 224])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("causal", [False, True])
def test_heads(dtype, d, page, causal):
    """Few rows, two blocks of them, many; tokens that end within a tile and a page."""
    Problem(dtype, 4, 2, d, [1, 3, 0, 2], [70, 33, 5, 0], page=page, causal=causal, seed=d, elsewhere=2.0).check()
    Problem(dtype, 6, 2, d, [9, 4], [140, 17], page=page, causal=causal, seed=d, elsewhere=2.0).check()
    Problem(dtype, 4, 2, d, [5, 60, 21], [70, 190, 33], page=page, causal=causal, seed=d, elsewhere=2.0).check()


@pytest.mark.parametrize("d", [136, 160, 192])
def test_windows(d):
    Problem("f32", 6, 2, d, [(7 * i) % 41 for i in range(10)], [(97 * i) % 500 for i in range(10)], page=16, causal=True, seed=d).check()
    Problem("f32", 2, 1, d, [520], [600], causal=True, seed=d).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("page", [0, 16])
def test_long_stretches_of_few_rows(dtype, d, page):
    """A wavefront walks one tile of tokens, two, three and many of them; more sequences than a stretch starts further on."""
    Problem(dtype, 2, 1, d, [1] * 5, [15, 33, 64, 257, 1000], page=page, seed=d, elsewhere=3.0).check()
    Problem(dtype, 2, 1, d, [1] * 120, [(211 * i) % 300 for i in range(120)], page=page, seed=d, elsewhere=3.0).check()
