"""`token_logprobs` of logits far from zero: finite masks of any size, whole rows of them, large positive logits, at temperatures around 1.

Tolerances are those of `test_gpu_logprobs` for log p and entropy: the exponents d = (x - max) / T carry three roundings however far
from zero x lies, since (x - max) c and x c - r are each rounded once beside c.  lse: max / T and its sum with log Z are rounded, 2 * 2^-24 of
what comes out (2e-7 |ref| allows more), and log Z as there.  What 32 bits do not hold is infinite."""
import math

import pytest

import readout_reference as R
from test_gpu_logprobs import call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MOST = torch.finfo(torch.float32).max
TEMPERATURES = [0.3, 0.7, 1.0, 1.5, 2.0]
SIZES = [3e5, 7.2e5, 7.4e5, 1e6, 1e9, 1e10, 1e12, 1e15, 1e20, 1e30]


def near(got, ref, flat, slope, what):
    if abs(ref) > MOST:
        assert got == math.copysign(math.inf, ref), (what, got, ref)
    else:
        assert abs(got - ref) <= flat + slope * abs(ref), (what, got, ref)


def check(x, temperature, tokens, top):
    o = call(x, temperature, tokens, top)
    torch.cuda.synchronize()
    o = {k: v.cpu() for k, v in o.items()}
    for r in range(x.shape[0]):
        ref = R.logprobs(x[r].double().cpu(), float(temperature[r]), int(tokens[r]), top)
        assert int(o["ranks"][r]) == ref["rank"] and o["top_tokens"][r].tolist() == ref["top_tokens"], r
        near(float(o["logprobs"][r]), ref["logprob"], 8e-6, 4e-7, ("logprob", r))
        near(float(o["entropy"][r]), ref["entropy"], 2e-5, 2e-6, ("entropy", r))
        near(float(o["lse"][r]), ref["lse"], 8e-6, 2e-7, ("lse", r))
        for got, want in zip(o["top_logprobs"][r].tolist(), ref["top_logprobs"]):
            near(got, want, 8e-6, 4e-7, ("top", r))


def rows_with(v, vocab, seed):
    """Ordinary logits with v in some places: everywhere, in front, behind, in the first chunk, every second chunk, every third token, all but one
    token, the first half, one token."""
    base = torch.randn(vocab, generator=torch.Generator().manual_seed(seed)) * 3
    i = torch.arange(vocab)
    places = [i >= 0, i < vocab - 30, i >= 30, i < 8, i // 8 % 2 == 0, i % 3 == 0, i != vocab // 2, i < vocab // 2, i == vocab - 5]
    return [torch.where(at, torch.tensor(v), base) for at in places]


def typed(rows, dtype):
    return torch.stack(rows).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)


def values(dtype):
    most = MOST if dtype == "f32" else torch.finfo(torch.bfloat16).max
    return [s * v for v in SIZES + [most] for s in (-1.0, 1.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", TEMPERATURES)
def test_in_one_workgroup(dtype, t):
    vocab = 2200
    x = typed([r for n, v in enumerate(values(dtype)) for r in rows_with(v, vocab, n)], dtype)
    tokens = (torch.arange(len(x)) * 37 % vocab).to(torch.int32).to(DEV)
    check(x, torch.full((len(x),), t, device=DEV), tokens, 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_in_slices(dtype, sign):
    """Masks that fill slices, beside slices that hold none."""
    vocab = 70000
    for n, v in enumerate(v for v in values(dtype) if v * sign > 0):
        x = typed(rows_with(v, vocab, n), dtype)
        tokens = (torch.arange(len(x)) * 9973 % vocab).to(torch.int32).to(DEV)
        check(x, torch.tensor([TEMPERATURES[(n + r) % 5] for r in range(len(x))], device=DEV), tokens, 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [2200, 70000])
def test_different_masks_in_one_row(dtype, vocab):
    """Sizes one after another, up and down, within a thread's chunks and within a chunk; and a largest logit on either side of every other."""
    n = vocab
    some = torch.tensor([-v for v in SIZES])
    rows = [some[torch.arange(n) // 8 % len(SIZES)], some[torch.arange(n) % len(SIZES)], some[len(SIZES) - 1 - torch.arange(n) * len(SIZES) // n],
            some[torch.arange(n) * len(SIZES) // n]]
    for v in (-1e6, -7.3e5, 7.3e5, 1e9):
        near_it = v + torch.arange(n) % 64 * abs(v) * 2.0 ** -20      # (a few units in the last place apart)
        rows += [near_it, torch.where(torch.arange(n) < n // 2, near_it, torch.tensor(-1e30))]
    x = typed(rows, dtype)
    tokens = (torch.arange(len(x)) * 501 % n).to(torch.int32).to(DEV)
    for t in TEMPERATURES:
        check(x, torch.full((len(x),), t, device=DEV), tokens, 4)
