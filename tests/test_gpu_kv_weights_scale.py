"""`accumulate_kv_weights` of few rows: the scale's rounding is no error of the score.

Tolerance.  Queries and keys have one channel, so their product is exact, and lse lies within 1 of the score: the exponent is a small number, rounded by 2^-25,
its second part by as little; the exponential is off by 2^-23, the factor of the rounded lse and its product by 2^-24 each: below 4 * 2^-23 =
4.8e-7.  A scale rounded to 24 bits would be off by up to 6e-8 of the score: 5e-6 at 80."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,scale", [(64, 0.0), (72, 0.0), (80, 0.0), (96, 0.0), (128, 0.0), (192, 0.0), (256, 0.0), (128, 0.1), (64, 0.3337)])
@pytest.mark.parametrize("queries,page", [(1, 0), (1, 16), (20, 16), (32, 0)])
def test_large_scores(dtype, d, scale, queries, page):
    from paper_2502_02534_amd import binding as B
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    exact = float(torch.tensor(scale)) if scale else 1 / math.sqrt(d)
    products = torch.tensor([3.0 * 2 ** i for i in range(8)] + [-3.0 * 2 ** i for i in range(8)], dtype=torch.float64)   # 3 to 384
    n = len(products)
    q, k = torch.zeros((n, queries, 1, d), dtype=t), torch.zeros((n, 16, 1, d), dtype=t)
    q[:, 0, 0, d // 2], k[:, :, 0, d // 2] = 3.0, (products / 3.0).to(t)[:, None]
    score = products * exact
    lse = torch.full((n, queries, 1), -math.inf)
    lse[:, 0, 0] = (score + 0.3).float()
    desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=1, num_kv_heads=1, head_dim=d, num_prompts=n, page_size=page,
                              causal=False, sm_scale=scale)
    out = torch.zeros((n, 1, 16), device=DEV)
    starts, pages = (i32(list(range(n + 1))), i32(list(range(n)))) if page else (i32([16 * b for b in range(n + 1)]), None)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    # (a page holds 16 tokens of the one KV head, one after another as contiguous ones do)
    B.accumulate_kv_weights(desc, q.to(DEV), k.to(DEV), i32([queries * b for b in range(n + 1)]), i32([16] * n), starts, pages, lse.to(DEV), n * queries,
                            queries, 16, 0.0, None, out, 16, ws)
    want = torch.exp(score - lse[:, 0, 0].double())
    err = ((out[:, 0].double().cpu() - want[:, None]).abs() / want[:, None]).amax(1)
    assert bool((err <= 4.8e-7).all()), list(zip(score.tolist(), err.tolist()))
