"""A decode loop with penalties that is run again: the history that a step's logits are shaped by is what this run has
drawn, not what an earlier one left in the record."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STEPS = 18


@pytest.fixture(scope="module")
def loop():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import prompt_to_samples
    return prompt_to_samples.run(prompt_lens=(40, 65), samples_per_prompt=3, steps=STEPS, vocab=3001, seed=11)["loop"]


def _restart(loop):
    loop.step.zero_()
    loop.finished.zero_()
    loop.sampler.tokens.fill_(-1)
    loop.attn.suffix_lens.zero_()


def test_a_second_run_draws_the_first_run_s_tokens(loop):
    first = loop.tokens_steps.clone()
    assert bool((first >= 0).all())
    for again in range(2):
        print(f"run {again + 2}", flush=True)
        _restart(loop)
        for _ in range(STEPS):
            loop.one_step()
        loop.flush()
        torch.cuda.synchronize()
        assert torch.equal(loop.tokens_steps, first)


def test_a_captured_step_that_starts_over_in_the_middle(loop):
    first = loop.tokens_steps.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.one_step()
    for steps in (7, 1, STEPS):
        print(f"{steps} steps", flush=True)
        _restart(loop)
        for _ in range(steps):
            graph.replay()
            _ = loop.attn.out.float().sum().item()  # eager work and a synchronisation between replays
        loop.flush()
        torch.cuda.synchronize()
        assert torch.equal(loop.tokens_steps[:steps], first[:steps])


def test_the_history_s_length_is_the_number_of_tokens_drawn(loop):
    """The shaped logits of a step by hand: with what the record holds before it, and nothing after."""
    from paper_2502_02534_amd import binding as B
    _restart(loop)
    raw, s = loop.raw_logits, loop.sampler
    for step in range(5):
        loop.one_step()
        torch.cuda.synchronize()
        got = s.logits.clone()
        lens = torch.full((raw.shape[0],), step, dtype=torch.int32, device=raw.device)
        history = loop.tokens_steps[:max(step, 1)].t()
        tensors = {k: v for k, v in loop._penalty_tensors.items() if k not in ("tokens", "token_lens")}
        pen = B.make_penalties(**tensors, tokens=history, token_lens=lens)
        B.penalize_logits(raw, B.SPD_BF16, raw.shape[0], raw.shape[1], raw.stride(0), pen, s.logits, s.logits.stride(0))
        torch.cuda.synchronize()
        assert torch.equal(got, s.logits)
