"""Every kernel of `token_logprobs`: batches of more rows than are cut into slices, of vocabularies around each kernel's limits, long rows whose lists the join
cannot hold at once.  A few rows of each against the definition, with the tolerances of `test_gpu_logprobs`."""
import math

import pytest

from test_gpu_logprobs import check

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"

# rows, vocabulary, alternatives
BATCHES = [(131, 2048, 64), (200, 8176, 5), (140, 8184, 20), (133, 8185, 20), (300, 8191, 7), (129, 8192, 64), (150, 8193, 5), (129, 32754, 64), (129, 32760, 3),
           (1030, 32768, 5), (129, 50257, 64), (140, 65529, 20), (131, 65537, 5), (1024, 128256, 5), (129, 131064, 64), (129, 131065, 64),
           (135, 140000, 0), (130, 262200, 20), (64, 128256, 20), (100, 128256, 20), (32, 131065, 64)]
LONG_LISTS = [(1, 1 << 19, 64), (2, (1 << 19) + 3, 63), (3, 600000, 40), (1, 1 << 20, 17)]


def batch(rows, vocab, dtype, pad, first, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    wide = torch.full((rows * (vocab + pad) + first,), float("nan"), dtype=t, device=DEV)
    x = wide[first:].view(rows, vocab + pad)[:, :vocab]
    for r in range(0, rows, 64):                                   # (in pieces: 1024 rows of 128256 at once are much)
        x[r:r + 64] = (torch.randn((min(64, rows - r), vocab), generator=g, device=DEV) * 3).to(t)
    # some rows are not of that kind: few different logits, masks in front, between and behind, equal ones
    i = torch.arange(vocab, device=DEV)
    x[1] = torch.randint(-2, 3, (vocab,), generator=g, device=DEV).to(t)
    x[2, : vocab - 100] = -math.inf
    x[3, i % 8 != 5] = -1e10
    x[4] = (-(i % 1000) * 0.25).to(t)
    x[5, 50:] = torch.finfo(t).min
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,first", [(0, 0), (3, 5)])
@pytest.mark.parametrize("rows,vocab,top", BATCHES)
def test_batches(dtype, pad, first, rows, vocab, top):
    x = batch(rows, vocab, dtype, pad, first, vocab + top)
    tokens = (torch.arange(rows, device=DEV) * 7919 % vocab).to(torch.int32)
    t = 0.3 + torch.rand(rows, generator=torch.Generator().manual_seed(rows)).to(DEV)
    t[5] = 1.0  # (the lowest value over less is no number of 32 bits)
    some = [0, 1, 2, 3, 4, 5, rows // 2, rows - 1] if vocab < 50000 and first == 0 else [1, 3, 5, rows - 1]
    check(x, t, tokens, top, rows=some)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,top", LONG_LISTS)
def test_lists_that_the_join_walks(dtype, rows, vocab, top):
    x = batch(8, vocab, dtype, 1, 0, vocab)
    for r in (0, 1, 5):
        part = x[r:r + rows]
        tokens = (torch.arange(part.shape[0], device=DEV) * 7919 % vocab).to(torch.int32)
        check(part, None, tokens, top, rows=[0])
