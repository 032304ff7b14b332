"""`token_logprobs` of given tokens whose logit is NaN."""
import math

import pytest

import readout_reference as R
from test_gpu_logprobs import call, near

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("vocab", [700, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_given_tokens_that_are_nan(vocab, dtype):
    """A NaN is a logit of -inf: no probability, behind all others."""
    x = torch.randn(3, vocab, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[:, 7] = float("nan")
    x[1, 30:50] = -math.inf
    x[2, 100:] = float("nan")
    tokens = torch.tensor([7, 7, 100], dtype=torch.int32, device=DEV)
    o = call(x.to(DEV), None, tokens, 4)
    clean = torch.where(x.isnan(), torch.tensor(-math.inf, dtype=x.dtype), x)
    for r in range(3):
        ref = R.logprobs(clean[r].double(), 1.0, int(tokens[r]), 4)
        assert int(o["ranks"][r]) == ref["rank"] and o["top_tokens"][r].tolist() == ref["top_tokens"]
        assert float(o["logprobs"][r]) == -math.inf
        near(float(o["entropy"][r]), ref["entropy"], 2e-5, 2e-6, r)
        near(float(o["lse"][r]), ref["lse"], 8e-6, 2e-7, r)
