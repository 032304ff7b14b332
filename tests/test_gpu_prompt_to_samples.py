"""The example that takes requests to sampled tokens, against the same thing done on the host: the prompts' attention,
the decode steps' attention over what the tables name, and greedy tokens from shaped logits."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def got():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import prompt_to_samples
    return prompt_to_samples.run(prompt_lens=(70, 203, 16), samples_per_prompt=3, steps=20, vocab=5003, seed=3)


def _bound(mass):
    # bf16: the result and the probabilities rounded to 8 significant bits each, and 2e-4 for scores in fp32
    return (2 * 2.0 ** -8 + 2e-4) * mass + 2e-3


def test_tables_deal_every_page_once(got):
    pages = got["prompt_tables"].page_indices.tolist() + got["sample_tables"].page_indices.tolist()
    assert pages == got["free"].tolist()[: len(pages)]
    assert got["prompt_tables"].new_indptr.tolist() == [0, 70, 273, 289]


def test_prompt_attention(got):
    q, k, v = (x.double().cpu() for x in got["qkv"])
    out = got["prompt_pass"].out.double().cpu()
    at = 0
    for n in got["prompt_lens"]:
        for h in range(q.shape[1]):
            s = q[at:at + n, h] @ k[at:at + n, h // 4].T / 128 ** 0.5
            s[torch.ones(n, n, dtype=torch.bool).triu(1)] = -torch.inf
            p = torch.softmax(s, 1)
            x = v[at:at + n, h // 4]
            assert bool(((out[at:at + n, h] - p @ x).abs() <= _bound(p @ x.abs())).all())
        at += n


def test_decode_attention_reads_what_the_prompt_pass_wrote(got):
    loop, (_, k, v) = got["loop"], got["qkv"]
    first = 0
    for b, n in enumerate(got["prompt_lens"]):
        for r in range(b * 3, b * 3 + 3):
            for step in (0, 7, 19):
                kk = torch.cat([k[first:first + n], loop.k_steps[: step + 1, r]]).double().cpu()
                vv = torch.cat([v[first:first + n], loop.v_steps[: step + 1, r]]).double().cpu()
                q = loop.q_steps[step, r].double().cpu()
                for h in (0, 13, 31):
                    p = torch.softmax(kk[:, h // 4] @ q[h] / 128 ** 0.5, 0)
                    want, mass = p @ vv[:, h // 4], p @ vv[:, h // 4].abs()
                    err = (loop.out_steps[step, r, h].double().cpu() - want).abs()
                    assert bool((err <= _bound(mass)).all()), (r, step, h, float(err.max()))
        first += n


def test_greedy_tokens_follow_the_penalties(got):
    """The highest shaped logit of every step, ties to the lowest index; a step may differ only where the two highest lie
    within 1e-5 of one another (the shaping rounds in fp32, logits are below 20)."""
    raw, s, tokens = got["raw"].double().cpu(), got["shaping"], got["loop"].tokens_steps.cpu()
    vocab = raw.shape[1]
    starts = got["prompt_tables"].new_indptr.tolist()
    repeats = 0
    for r in range(raw.shape[0]):
        b = r // got["samples_per_prompt"]
        prompt = torch.zeros(vocab, dtype=torch.bool)
        prompt[got["prompt_tokens"][starts[b]:starts[b + 1]].long().cpu()] = True
        count = torch.zeros(vocab, dtype=torch.float64)
        for step in range(tokens.shape[0]):
            x = raw[r].clone()
            rho = float(s["repetition"][r])
            seen = prompt | (count > 0)
            x = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
            x = x - float(s["frequency"][r]) * count - float(s["presence"][r]) * (count > 0)
            x[int(s["bias_tokens"][r])] += 2.5
            if r % 2 == 0:
                half = (-(-vocab // 32)) // 2 * 32
                odd = torch.arange(vocab) % 2 == 1
                x[odd & (torch.arange(vocab) < half)] = -torch.inf
            top = torch.topk(x, 2)
            t = int(tokens[step, r])
            assert t == int(top.indices[0]) or float(top.values[0] - x[t]) <= 1e-5, (r, step)
            repeats += int(count[t] > 0)
            count[t] += 1
    assert repeats > 0  # (the penalties were at work on tokens drawn more than once)


def test_a_loop_without_penalties_is_as_before(got):
    from paper_2502_02534_amd import device as D
    loop = got["loop"]
    with pytest.raises(ValueError):
        D.DecodeLoop(loop.attn, loop.sampler, loop.q_steps, loop.k_steps, loop.v_steps, loop.u_steps, raw_logits=got["raw"])
    with pytest.raises(ValueError):
        D.DecodeLoop(loop.attn, loop.sampler, loop.q_steps, loop.k_steps, loop.v_steps, loop.u_steps, one_launch=False,
                     raw_logits=got["raw"], penalties=got["shaping"])
    plain = D.DecodeLoop(loop.attn, loop.sampler, loop.q_steps, loop.k_steps, loop.v_steps, loop.u_steps)
    assert plain.penalties is None
