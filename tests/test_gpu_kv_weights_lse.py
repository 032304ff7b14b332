"""`accumulate_kv_weights`: the log-sum-exp of a row is an error that all of its tokens share, so it must not be rounded by more than the weights are.

Tolerance.  A query of zeros has scores of exactly 0, and every token's weight is exp(-lse).  The exponential of the rounded exponent is off by
2^-23; what the rounding took is a factor next to 1, itself rounded (2^-24); the product with it and the sum over the one row that counts, 2^-24
each; 2^-23 for the second order: below 4 * 2^-23 = 4.8e-7.  Rounding lse log2(e) to 24 bits alone would be up to 2.6e-6 at lse 50."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LSES = [0.1, 0.7, 1.0, 3.3, 9.017, 12.34, 20.5, 33.3, 45.45, 50.1, 60.7, 70.07, 80.9, -0.3, -5.3, -40.2, -71.9]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("queries,g,tokens", [(1, 1, 40), (5, 4, 40), (20, 3, 300), (300, 1, 70), (2000, 1, 33)])
def test_a_rows_log_sum_exp(dtype, page, d, queries, g, tokens):
    """Few rows, some more, many, and (where parts pay) rows in parts; one of them counts."""
    from paper_2502_02534_amd import binding as B
    n = len(LSES) if queries < 2000 else 1
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    held = -(-tokens // 16)
    desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=g, num_kv_heads=1, head_dim=d, num_prompts=n, page_size=page,
                              causal=False)
    q = torch.zeros((n * queries, g, d), dtype=t, device=DEV)
    k = torch.randn((n * held, 1, 16, d) if page else (n * tokens, 1, d), device=DEV).to(t)
    starts, pages = i32([held * b for b in range(n + 1)]) if page else i32([tokens * b for b in range(n + 1)]), i32(list(range(n * held))) if page else None
    ws = torch.empty(max(256, B.accumulate_kv_weights_workspace_size(desc, n * queries, queries, tokens)), dtype=torch.uint8, device=DEV)
    for first in range(0, len(LSES), n):
        some = torch.tensor(LSES[first:first + n], device=DEV)
        lse = torch.full((n, queries, g), -math.inf, device=DEV)
        for b in range(n):
            lse[b, (7 * b + first) % queries, b % g] = some[b]
        out = torch.zeros((n, 1, tokens), device=DEV)
        B.accumulate_kv_weights(desc, q, k, i32([queries * b for b in range(n + 1)]), i32([tokens] * n), starts, pages, lse, n * queries, queries, tokens, 0.0,
                                None, out, tokens, ws)
        want = torch.exp(-some.double())[:, None, None]
        err = ((out.double() - want).abs() / want).amax((1, 2))
        assert bool((err <= 4.8e-7).all()), list(zip(some.tolist(), err.tolist()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries", [3, 50])
def test_log_sum_exps_of_any_size(dtype, queries):
    """Far ones, infinite ones and the type's lowest value: a weight of 0 or infinity, and no NaN."""
    from paper_2502_02534_amd import binding as B
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    some = [-math.inf, math.inf, 1e3, -1e3, 3e7, -3e7, 1e12, -1e12, 3e38, -3e38]
    n = len(some)
    desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=1, num_kv_heads=1, head_dim=64, num_prompts=n, causal=False)
    q, k = torch.randn((n * queries, 1, 64), device=DEV).to(t), torch.randn((n * 20, 1, 64), device=DEV).to(t)
    lse = torch.tensor(some, device=DEV)[:, None].expand(n, queries).contiguous()
    out = torch.zeros((n, 1, 20), device=DEV)
    ws = torch.empty(max(256, B.accumulate_kv_weights_workspace_size(desc, n * queries, queries, 20)), dtype=torch.uint8, device=DEV)
    B.accumulate_kv_weights(desc, q, k, i32([queries * b for b in range(n + 1)]), i32([20] * n), i32([20 * b for b in range(n + 1)]), None, lse, n * queries, queries,
                            20, 0.0, None, out, 20, ws)
    for b, x in enumerate(some):
        want = 0.0 if x > 0 or x == -math.inf else math.inf
        assert bool((out[b] == want).all()), (x, out[b])
