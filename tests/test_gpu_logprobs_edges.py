"""`token_logprobs` at temperatures whose quotient with 1 does not fit, or hardly."""
import math

import pytest

import readout_reference as R
from test_gpu_logprobs import call
from test_gpu_logprobs_far import near

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("vocab", [700, 40000])
@pytest.mark.parametrize("t", [1e-45, 1e-40, 3e-39, 1.2e-38])
def test_temperatures_next_to_zero(vocab, t):
    """1 / T is infinite below 2.9e-39.  The largest logits have all of the probability, whatever their sign, zero among them."""
    x = torch.randn(4, vocab, generator=torch.Generator().manual_seed(1)) - 9.0
    x[0, 17] = x[0, 23] = 0.0
    x[1, 5] = 3.0
    x[2, 8] = -1e-3
    x[3] = 0.0
    tokens = torch.tensor([23, 5, 8, 2], dtype=torch.int32, device=DEV)
    o = call(x.to(DEV), torch.full((4,), t, device=DEV), tokens, 3)
    most = [2, 1, 1, vocab]
    for r in range(4):
        near(float(o["logprobs"][r]), -math.log(most[r]), 8e-6, 4e-7, r)
        near(float(o["entropy"][r]), math.log(most[r]), 2e-5, 2e-6, r)
    assert o["top_tokens"].tolist() == [R.logprobs(row.double(), 1.0, 0, 3)["top_tokens"] for row in x]
    held = float(torch.tensor(t))
    for r in range(4):
        near(float(o["lse"][r]), float(x[r].max()) / held + math.log(most[r]), 8e-6, 2e-7, r)
