"""`prompt_attn` on scores of any finite size: those whose differences alone matter (2^31 and more, where a unit in the last
place is larger than an exponent may be), all of them far below zero, and a row's first scores far below its later ones.

Queries and keys are powers of two, so that scores are exact and equal ones are equal to the last bit: a row's result is
the mean of the values of its highest tokens, every other token's probability being 0 in 64 bits too (the next score is
at least 2^20 lower).  Tolerances: bf16 2^-8 for the result, 2^-8 for the probabilities, of the mean magnitude, fp32 1e-5 of it,
1e-6 for results near zero.  The log-sum-exp is the score and a small logarithm: the scale in base 2, the product, the way back and the
sum round four times, 8 * 2^-24 of its size allows two units each."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_prompt_attn import PAGE, Problem  # noqa: E402

pytestmark = pytest.mark.gpu


def _check(p, score_of):
    """score_of[b][t]: what the score of token t of prompt b is, for every query."""
    out, lse = p.run()
    for b, n in enumerate(p.new):
        first, L = int(p.query_indptr[b]), p.kv[b]
        s, v = score_of[b].double(), p.rows_of(b, "v").double()
        for i in range(n):
            if n > 100 and i % 13 and i < n - 3:
                continue
            see = L - n + i + 1 if p.causal else L
            top = s[:see] == s[:see].max()
            got, got_lse = out[first + i].double(), lse[first + i].double()
            want_lse = s[:see].max() + math.log(int(top.sum()))
            assert bool(((got_lse - want_lse).abs() <= 8 * 2.0 ** -24 * want_lse.abs() + 1e-5).all()), (b, i, got_lse, want_lse)
            x = v[:see][top]                                                   # [tokens, KV heads, channels]
            want, mass = (y.mean(0).repeat_interleave(p.hq // p.hkv, 0) for y in (x, x.abs()))
            tol = (2 * 2.0 ** -8 if p.dtype == "bf16" else 1e-5) * mass + 1e-6
            assert bool(((got - want).abs() <= tol).all()), (b, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("new,past,page", [([1], [0], 0), ([1, 40], [0, 0], PAGE), ([70, 9], [0, 300], 0),   # single tiles and edges
                                           ([300, 1100], [0, 0], 0), ([260], [40], PAGE),                  # long stretches
                                           ([1, 3], [1500, 700], PAGE), ([5], [2000], 0)])               # parts
@pytest.mark.parametrize("size", [2.0 ** 33, 2.0 ** 60, 2.0 ** 110])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(dtype, d, new, past, page, size, sign):
    hq = 16 if max(new) > 1000 else 4  # (enough units to need no parts)
    p = Problem(dtype, hq, 2, d, new, past, page=page, seed=d, scale=1.0)
    # q = sqrt(size), k = +-sqrt(size) * (1 + t % 5) / 8 in one channel: scores +-size (1 + t % 5) / 8
    root = 2.0 ** (math.log2(size) // 2)
    p.q.zero_()
    p.q[..., 7] = root
    scores = []
    for b, L in enumerate(p.kv):
        steps = (1 + torch.arange(L) * 7 % 5).double() / 8 * sign
        k = torch.zeros(L, 2, d)
        k[..., 7] = (steps * (size / root))[:, None].float()
        at = int(p.kv_indptr[b])
        if page:
            for t in range(L):
                p.k[p.pages[at + t // PAGE], :, t % PAGE] = k[t].to(p.k.dtype)
        else:
            p.k[at:at + L] = k.to(p.k.dtype)
        scores.append(steps * size)
    print(f"large scores {dtype} {d} {new} {past} {sign * size:g}", flush=True)
    _check(p, scores)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,past", [([500], [0]), ([3], [1300])])
def test_scores_that_grow_and_fall(dtype, d, new, past):
    """From -2^100 up to 2^100 and down again along the tokens, in stretches of 48."""
    p = Problem(dtype, 16, 2, d, new, past, seed=d, scale=1.0)
    L = p.kv[0]
    ladder = [-2.0 ** 100, -2.0 ** 70, -2.0 ** 34, 0.0, 2.0 ** 34, 2.0 ** 70, 2.0 ** 100, 2.0 ** 50, -2.0 ** 90]
    s = torch.tensor([ladder[t // 48 % len(ladder)] for t in range(L)], dtype=torch.float64)
    p.q.zero_()
    p.k.zero_()
    p.q[..., 5] = 2.0 ** 50
    p.k[..., 5] = (s / 2.0 ** 50).to(p.k.dtype)[:, None]
    _check(p, [s])
