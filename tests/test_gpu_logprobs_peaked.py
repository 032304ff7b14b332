"""Entropy of rows that few logits dominate, from `token_logprobs`.

Tolerance.  Two logits of a row count, the larger one and one `gap` below it; two lie 2^23.5 below, all others are masked.  In base 2 and units of
2^-24: the exponentials are off by 2, which a term's own p and 1 + |y| <= 2 weigh (4); up to four additions that are rounded in Z, and four in S, of
numbers below 2 (8); the logarithm (2), the quotient and the difference (2).  16 * 2^-24 * ln 2 = 6.6e-7.  Sums whose numbers are 24 times
as large while they are made are off by more."""
import math

import pytest

from test_gpu_logprobs import call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [6000, 50000, 128256])
def test_entropy(dtype, vocab):
    g = torch.Generator().manual_seed(vocab)
    rows = []
    for n in range(200):
        x = torch.full((vocab,), -math.inf)
        top, gap = 4 + 8 * float(torch.rand(1, generator=g)), 0.5 + 5 * float(torch.rand(1, generator=g))
        place = int(torch.randint(4200, vocab - 16, (1,), generator=g))
        x[place - 4096] = x[place - 2048] = top - 16.3          # (some chunks earlier)
        x[place] = top
        x[place + n % 9 + 1] = top - gap
        rows.append(x)
    x = torch.stack(rows).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
    tokens = torch.zeros(200, dtype=torch.int32, device=DEV)
    for each in (200, 20):                                       # a workgroup a row, and in slices
        entropy = torch.cat([call(x[i:i + each], None, tokens[i:i + each], 0)["entropy"] for i in range(0, 200, each)]).cpu()
        worst = 0.0
        for r in range(200):
            y = x[r].double().cpu()
            logp = torch.log_softmax(y[y > -math.inf], 0)
            worst = max(worst, abs(float(entropy[r]) + float((logp.exp() * logp).sum())))
        assert worst <= 6.6e-7, (each, worst)
