"""The example of long generations in a bounded cache, against the same thing done on the host: the prompts' weights and the half of
them that stays, every step's attention over what was kept, the samples' weights and what they kept of their own tokens, and the
log probabilities of what was drawn."""
import math
import os
import sys

import pytest

import readout_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SCALE = 1 / math.sqrt(128)


@pytest.fixture(scope="module")
def got():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import bounded_samples
    return bounded_samples.run(prompt_lens=(70, 203, 16), samples_per_prompt=2, steps=61, room=32, budget=14, sinks=1, recent=5, vocab=5003,
                               seed=3)


def test_weights_and_halves_of_the_prompts(got):
    q, k, _ = (x.double().cpu() for x in got["qkv"])
    weights = got["weights"].cpu()
    at = 0
    for b, n in enumerate(got["prompt_lens"]):
        for j in range(8):
            total = torch.zeros(n, dtype=torch.float64)
            for h in range(4 * j, 4 * j + 4):
                s = q[at:at + n, h] @ k[at:at + n, j].T * SCALE
                s[torch.ones(n, n, dtype=torch.bool).triu(1)] = -torch.inf
                total += torch.softmax(s, 1).sum(0)
            # (the attention's own log-sum-exps are within 1e-4 of the exact ones, which every term shares; scores below 60)
            assert bool(((weights[b, j, :n].double() - total).abs() <= 1.4e-4 * total).all())
            want = R.kept(weights[b, j, :n].tolist(), n, got["kept"][b], got["sinks"], got["recent"])
            assert got["source"][b, j, :len(want)].tolist() == want
        at += n
    assert got["prefix_lens"].tolist() == got["kept"]


def test_every_step(got):
    """Attention over the kept prompt and the kept tokens of the sample, whose weights add up to what its heads gave them."""
    loop = got["loop"]
    q, k, v = (x.double().cpu() for x in (loop.q_steps, loop.k_steps, loop.v_steps))
    _, pk, pv = (x.double().cpu() for x in got["qkv"])
    out, lens = loop.out_steps.double().cpu(), loop.lens_steps.cpu()
    starts = [0, 70, 273]
    evictions = {e[0]: [x.cpu() for x in e[1:]] for e in got["evictions"]}
    assert sorted(evictions) == [32, 50]
    for r in range(out.shape[1]):
        b = r // got["samples_per_prompt"]
        for j in range(8):
            src = [starts[b] + t for t in got["source"][b, j, :got["kept"][b]].tolist()]
            prefix_k, prefix_v = pk[src, j], pv[src, j]
            held, weights = [], []
            for step in range(out.shape[0]):
                if step in evictions:
                    mine, source, new = evictions[step]
                    for x, w in zip(mine[r, j, :len(held)].tolist(), weights):
                        assert abs(x - w) <= 2e-4 * w + 1e-30, (step, x, w)  # (as above, and up to 32 sums)
                    want = R.kept(mine[r, j].tolist(), len(held), got["budget"], got["sinks"], got["recent"])
                    assert source[r, j].tolist() == want and int(new[r]) == len(want)
                    held, weights = [held[t] for t in want], [weights[t] for t in want]
                held.append(step)
                weights.append(0.0)
                assert int(lens[step, r]) == (got["budget"] if step + 1 in evictions else len(held))  # (as the next step found it)
                own_k, own_v = k[held, r, j], v[held, r, j]
                s = torch.cat([prefix_k, own_k]) @ q[step, r, 4 * j:4 * j + 4].T * SCALE
                p = torch.softmax(s, 0)
                values = torch.cat([prefix_v, own_v])
                ref, mass = p.T @ values, p.T @ values.abs()
                err = (out[step, r, 4 * j:4 * j + 4] - ref).abs()
                assert bool((err <= (2 * 2.0 ** -8 + 2e-4) * mass + 2e-3).all()), (r, j, step)
                own = p[len(src):].sum(1).tolist()
                weights = [w + x for w, x in zip(weights, own)]


def test_log_probabilities(got):
    loop, logits = got["loop"], got["logits"].double().cpu()
    for step in (0, 17, 32, 60):
        for r in range(logits.shape[0]):
            token = int(loop.tokens_steps[step, r])
            ref = R.logprobs(logits[r], 0.800000011920929, token, got["num_top"])
            assert abs(float(loop.logprobs_steps[step, r]) - ref["logprob"]) <= 8e-6 + 4e-7 * abs(ref["logprob"])
            assert int(loop.ranks_steps[step, r]) == ref["rank"]
            assert abs(float(loop.entropy_steps[step, r]) - ref["entropy"]) <= 2e-5 + 2e-6 * ref["entropy"]
            assert loop.top_tokens_steps[step, r].tolist() == ref["top_tokens"]
            for x, y in zip(loop.top_logprobs_steps[step, r].tolist(), ref["top_logprobs"]):
                assert abs(x - y) <= 8e-6 + 4e-7 * abs(y)
