"""Decode loops that report log probabilities and accumulate weights: the same tokens and outputs as loops that do neither, step by step
and in one launch, and weights that are forgotten when the loop starts over."""
import copy

import numpy as np
import pytest

from paper_2502_02534_amd import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

STEPS, VOCAB = 6, 3001


@pytest.fixture(scope="module")
def dev():
    from paper_2502_02534_amd import binding, device
    binding.load()
    return device


def _loop(dev, dtype, one_launch, num_top, said, budget, room=40):
    spec = W.small_spec(dtype=dtype, num_q_heads=8, num_kv_heads=2, head_dim=128 if dtype == "bf16" else 64, num_prompts=2,
                        samples_per_prompt=3, prefix_len=(30, 90), suffix_len=(0, 20))
    inp = W.make_attn_inputs(0, spec=spec, seed=5)
    n = inp.q.shape[0]
    inp = copy.copy(inp)
    wide = lambda x: np.concatenate([x, np.zeros((n, room - x.shape[1]) + x.shape[2:], x.dtype)], 1)  # noqa: E731
    inp.k_suffix, inp.v_suffix, inp.max_suffix_len = wide(inp.k_suffix), wide(inp.v_suffix), room
    attn = dev.upload_attn(inp)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda:0")  # noqa: E731
    logits = normal(n, VOCAB) * 3
    from paper_2502_02534_amd import binding as B
    sampler = dev.DeviceSampler(logits, torch.full((n,), 0.7, device="cuda:0"), torch.full((n,), 0.9, device="cuda:0"), torch.zeros(n, device="cuda:0"),
                                torch.empty(n, dtype=torch.int32, device="cuda:0"),
                                torch.empty(B.sample_tokens_workspace_size(n, VOCAB), dtype=torch.uint8, device="cuda:0"))
    t = attn.q.dtype
    hq, d, hkv = attn.q.shape[1], attn.q.shape[2], attn.desc.num_kv_heads
    logprobs = dev.DeviceLogprobs(logits, sampler.tokens, sampler.temperature, num_top) if said else None
    eviction = dev.DeviceEviction(attn, budget, 1, 4) if budget else None
    return dev.DecodeLoop(attn, sampler, normal(STEPS, n, hq, d).to(t), normal(STEPS, n, hkv, d).to(t), normal(STEPS, n, hkv, d).to(t),
                          torch.rand((STEPS, n), generator=g, device="cuda:0"), one_launch=one_launch, logprobs=logprobs, eviction=eviction)


def _run(loop):
    for _ in range(STEPS):
        loop.one_step()
    loop.flush()
    torch.cuda.synchronize()
    return loop


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("one_launch", [True, False])
@pytest.mark.parametrize("num_top", [0, 4])
def test_loops_that_report_draw_the_same(dev, dtype, one_launch, num_top):
    plain, full = _run(_loop(dev, dtype, one_launch, 0, False, 0)), _run(_loop(dev, dtype, one_launch, num_top, True, 16))
    for name in ("tokens_steps", "out_steps", "lens_steps"):
        assert torch.equal(getattr(plain, name), getattr(full, name)), name
    logp = torch.log_softmax(full.logprobs.logits.double() / 0.699999988079071, 1)
    for step in range(STEPS):
        want = logp.gather(1, full.tokens_steps[step].long()[:, None])[:, 0]
        assert bool(((full.logprobs_steps[step] - want).abs() <= 8e-6 + 4e-7 * want.abs()).all())
        if num_top:
            assert torch.equal(full.top_tokens_steps[step].long(), logp.topk(num_top, 1)[1])  # (no ties among random logits)
    assert hasattr(full, "top_tokens_steps") == bool(num_top)
    # a sample's weights and what its prompt got add up to its query heads: here the suffix's share, below it
    total = full.eviction.weights.sum((1, 2))
    assert bool((total > 0).all()) and bool((total <= 8.0 * STEPS * 1.001).all())
    tail = torch.arange(full.eviction.weights.shape[2], device="cuda:0") >= full.attn.suffix_lens[:, None, None]
    assert float(full.eviction.weights[tail.expand_as(full.eviction.weights)].abs().sum()) == 0.0


def test_reset(dev):
    loop = _run(_loop(dev, "bf16", True, 0, False, 16))
    assert float(loop.eviction.weights.sum()) > 0
    loop.eviction.reset()
    assert float(loop.eviction.weights.abs().sum()) == 0.0
    # suffixes longer than the budget shrink to it, shorter ones stay
    before = loop.attn.suffix_lens.clone()
    loop.eviction.evict()
    assert torch.equal(loop.attn.suffix_lens, before.clamp(max=16))
