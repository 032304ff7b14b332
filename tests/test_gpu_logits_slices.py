"""`penalize_logits` at the sizes that take longer slices of the vocabulary (from 3 and from 12 million logits on), and where
a slice holds more different tokens than its table of counts, against the definition in 64 bits.  Reference and tolerances are
those of tests/test_gpu_logits.py."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_logits import Case  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(25, 128256), (31, 100001), (100, 128256), (123, 100003), (65, 50257), (250, 50257)])
def test_every_part_in_longer_slices(dtype, rows, vocab):
    Case(rows, vocab, dtype, seed=rows, gen=300, pad=rows % 4, by_step=rows % 2 == 0).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 30, 100])
def test_no_part_in_longer_slices(dtype, rows):
    Case(rows, 128256, dtype, seed=rows, parts="").check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,crowd", [(3, 9001, 9001),           # slices of 4096
                                              (25, 128256, 20000),       # of 8192
                                              (100, 128256, 40000)])     # of 16384
def test_more_different_tokens_than_a_slice_s_table_holds(dtype, rows, vocab, crowd):
    """Histories that name every one of the first `crowd` tokens, some twice: any slice of them has more than 2048."""
    c = Case(rows, vocab, dtype, seed=crowd, parts="rfpmbg", pad=1)
    g = torch.Generator().manual_seed(crowd)
    row = torch.cat([torch.randperm(crowd, generator=g), torch.randint(0, crowd, (500,), generator=g)]).tolist()
    c.tokens, c.lens = [row] * rows, [0 if r > 3 else len(row) if r % 3 else len(row) - 700 for r in range(rows)]
    c.by_step = rows == 25
    c.check()


def test_the_crowd_through_biases_too():
    """A table that the history fills to the last place, and one token more from the biases."""
    for extra in (0, 1):
        c = Case(2, 9000, "f32", seed=extra, parts="fp")
        row = list(range(0, 4096, 2))                                    # 2048 tokens of the first slice
        c.tokens, c.lens = [row, row], [2048, 2047]
        c.biases = [[(4095, 1.5)] * extra, [(4095, -2.5)] * extra]
        c.check()
