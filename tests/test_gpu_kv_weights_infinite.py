"""`accumulate_kv_weights` of infinite scores: exp of -inf is 0 and of +inf is +inf, whatever the scale's second part is, and only for the token that has
such a key."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,scale", [(64, 0.0), (80, 0.0), (128, 0.0), (256, 0.0), (64, 0.3337), (64, 0.25 / 1.4426950408889634)])
@pytest.mark.parametrize("queries", [1, 20, 70])
def test_infinite_keys(dtype, d, scale, queries):
    from paper_2502_02534_amd import binding as B
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    g = torch.Generator().manual_seed(d)
    q, k = torch.randn((queries, 1, d), generator=g).to(t), torch.randn((50, 1, d), generator=g).to(t)
    q[:, 0, 3] = 1.0
    k[7, 0, 3], k[20, 0, 3], k[49, 0, 3] = -math.inf, math.inf, -math.inf
    lse = torch.full((queries, 1), 6.0)
    desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=1, num_kv_heads=1, head_dim=d, num_prompts=1, causal=False,
                              sm_scale=scale)
    out = torch.zeros((1, 1, 50), device=DEV)
    ws = torch.empty(max(256, B.accumulate_kv_weights_workspace_size(desc, queries, queries, 50)), dtype=torch.uint8, device=DEV)
    B.accumulate_kv_weights(desc, q.to(DEV), k.to(DEV), i32([0, queries]), i32([50]), i32([0, 50]), None, lse.to(DEV), queries, queries, 50, 0.0, None, out, 50, ws)
    out = out[0, 0].cpu()
    assert out[7] == 0.0 and out[20] == math.inf and out[49] == 0.0
    others = [i for i in range(50) if i not in (7, 20, 49)]
    want = torch.exp(k[others, 0].double() @ q[:, 0].double().T * (float(torch.tensor(scale)) if scale else 1 / math.sqrt(d)) - 6.0).sum(1)
    assert bool(((out[others].double() - want).abs() <= 3e-5 * want).all())
