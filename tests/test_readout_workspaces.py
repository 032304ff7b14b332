"""A workspace that is sized once, for the largest call, is enough for every smaller one: fewer rows or queries are cut into more parts
(host arithmetic: no GPU needed)."""
import os
import random

import pytest

from test_sanitizers import ROOT, _build_and_run


@pytest.fixture(scope="module")
def B():
    from paper_2502_02534_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    binding.load()
    return binding


@pytest.mark.parametrize("vocab", [1000, 32000, 50257, 128256, 1 << 18, 1 << 20])
@pytest.mark.parametrize("top", [0, 20])
def test_log_probabilities(B, vocab, top):
    size = B.token_logprobs_workspace_size
    for most in (1, 64, 128, 129, 1024, 5000):
        largest = size(most, vocab, top)
        assert max(size(rows, vocab, top) for rows in range(0, most + 1, max(1, most // 200))) <= largest
        assert size(most, vocab // 3, top // 2) <= largest


@pytest.mark.parametrize("dtype", [0, 1])
def test_weights(B, dtype):
    rng = random.Random(dtype)
    desc = lambda n: B.make_prompt_desc(dtype=dtype, num_q_heads=32, num_kv_heads=8, head_dim=128, num_prompts=n)  # noqa: E731
    size = B.accumulate_kv_weights_workspace_size
    assert size(desc(4), 512, 512, 4096) <= size(desc(4), 2048, 512, 4096)
    for _ in range(300):
        n, query, kv = rng.randint(1, 40), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 15))
        largest = size(desc(n), n * query, query, kv)
        for _ in range(40):
            m, a, b = rng.randint(1, n), rng.randint(0, query), rng.randint(0, kv)
            assert 0 < size(desc(m), rng.randint(0, m * a), a, b) <= largest, (n, query, kv, m, a, b)


def test_sizes_hold_for_every_plan(tmp_path):
    """What a call asks for, against the size that a larger one's query says, under the sanitizers."""
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "readout_workspace_driver.cpp")], ["-std=c++17"])
    assert out.startswith("ok")
