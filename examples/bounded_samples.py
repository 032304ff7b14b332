"""Long generations in a bounded cache, all on the device: the prompts' attention says which of their tokens are used, the
samples decode from the half that is (the whole prompts stay where they are, for others), and every sample's own tokens are
kept within a few pages by their accumulated weight while it generates more than these hold.  Every step reports how probable the
drawn token was, the entropy and the alternatives.

Keys, queries, values and logits are random (there are no weights here); everything else is what a server does.

    python examples/bounded_samples.py [--steps 96]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2502_02534_amd import binding as B  # noqa: E402
from paper_2502_02534_amd import device as D  # noqa: E402

HQ, HKV, HEAD_DIM, PAGE = 32, 8, 128, 16


def _i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def run(prompt_lens=(700, 1203, 64), samples_per_prompt=4, steps=96, room=64, budget=32, sinks=2, recent=16, vocab=32000, num_top=3, seed=0,
        dev="cuda:0"):
    """Returns what a test needs.  room: tokens that a sample's pages hold; budget: those that stay when they are full."""
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)  # noqa: E731
    prompts, rows, tokens = len(prompt_lens), len(prompt_lens) * samples_per_prompt, sum(prompt_lens)

    # pages: for the prompts, for what the samples see of them, for the samples' own tokens
    kept = [max(1, n // 2) for n in prompt_lens]
    pages = lambda lens: sum(-(-n // PAGE) for n in lens)  # noqa: E731
    pool = (pages(prompt_lens) + pages(kept) + rows * -(-room // PAGE), HKV, PAGE, HEAD_DIM)
    k_pool, v_pool = (torch.zeros(pool, dtype=torch.bfloat16, device=dev) for _ in range(2))
    free = torch.randperm(pool[0], generator=g, device=dev).to(torch.int32)
    prompt_tables = D.build_tables(_i32(prompt_lens, dev), free, pages(prompt_lens), tokens)
    kept_tables = D.build_tables(_i32(kept, dev), free, pages(kept), free_begin=prompt_tables.free_end)
    sample_tables = D.build_tables(torch.full((rows,), room, dtype=torch.int32, device=dev), free, rows * -(-room // PAGE),
                                   free_begin=kept_tables.free_end)

    # 1. the prompts' own attention, and what each of their tokens got of it
    q, k, v = normal(tokens, HQ, HEAD_DIM), normal(tokens, HKV, HEAD_DIM), normal(tokens, HKV, HEAD_DIM)
    longest = max(prompt_lens)
    prompt_pass = D.DevicePrompts(prompt_tables, q, k, v, k_pool, v_pool, longest, longest)
    prompt_pass.run()
    weights = torch.zeros((prompts, HKV, longest), device=dev)
    ws = torch.empty(max(256, B.accumulate_kv_weights_workspace_size(prompt_pass.desc, tokens, longest, longest),
                         B.select_kv_tokens_workspace_size(prompts, HKV, longest)), dtype=torch.uint8, device=dev)
    B.accumulate_kv_weights(prompt_pass.desc, q, k_pool, prompt_tables.packed_indptr, prompt_tables.packed_lens, prompt_tables.page_indptr,
                            prompt_tables.page_indices, prompt_pass.lse, tokens, longest, longest, 0.0, None, weights, longest, ws)

    # 2. half of each prompt, in pages of its own
    source = torch.zeros((prompts, HKV, max(kept)), dtype=torch.int32, device=dev)
    kept_lens, prefix_lens = torch.zeros(prompts, dtype=torch.int32, device=dev), torch.zeros(prompts, dtype=torch.int32, device=dev)
    B.select_kv_tokens(weights, longest, prompts, HKV, prompt_tables.lens, longest, _i32(kept, dev), max(kept), sinks, recent, source,
                       source.stride(1), kept_lens, ws)
    B.compact_kv(prompt_pass.desc, source, source.stride(0), source.stride(1), kept_lens, max(kept), prompt_tables.page_indptr,
                 prompt_tables.page_indices, k_pool, v_pool, kept_tables.page_indptr, kept_tables.page_indices, k_pool, v_pool, None, None, 0,
                 prefix_lens)

    # 3. decode: attention over that half and over the sample's own tokens, greedy sampling, its log probabilities
    desc = B.make_desc(dtype=B.SPD_BF16, num_q_heads=HQ, num_kv_heads=HKV, head_dim=HEAD_DIM, num_prompts=prompts, num_samples=rows,
                       max_samples_per_prompt=samples_per_prompt, page_size=PAGE)
    attn_ws = torch.empty(B.shared_prefix_decode_attn_workspace_size(desc, max(kept), room), dtype=torch.uint8, device=dev)
    sample_indptr = _i32([i * samples_per_prompt for i in range(prompts + 1)], dev)
    attn = D.DeviceAttn(desc, normal(rows, HQ, HEAD_DIM), k_pool, v_pool, prefix_lens, kept_tables.page_indptr, kept_tables.page_indices,
                        sample_indptr, k_pool, v_pool, torch.zeros(rows, dtype=torch.int32, device=dev), sample_tables.page_indptr,
                        sample_tables.page_indices, max(kept), room, normal(rows, HQ, HEAD_DIM), torch.empty((rows, HQ), device=dev), attn_ws)
    logits = torch.randn((rows, vocab), generator=g, device=dev) * 3
    sampler = D.DeviceSampler(logits, torch.full((rows,), 0.8, device=dev), torch.ones(rows, device=dev), torch.zeros(rows, device=dev),
                              torch.empty(rows, dtype=torch.int32, device=dev),
                              torch.empty(B.sample_tokens_workspace_size(rows, vocab), dtype=torch.uint8, device=dev))
    logprobs = D.DeviceLogprobs(logits, sampler.tokens, sampler.temperature, num_top)
    eviction = D.DeviceEviction(attn, budget, sinks, recent)
    u_steps = torch.rand((steps, rows), generator=g, device=dev)
    loop = D.DecodeLoop(attn, sampler, normal(steps, rows, HQ, HEAD_DIM), normal(steps, rows, HKV, HEAD_DIM),
                        normal(steps, rows, HKV, HEAD_DIM), u_steps, end_token=-2,  # (a token that is never drawn)
                        logprobs=logprobs, eviction=eviction)

    # one step as it is, the rest replayed from one captured step; room is made whenever the samples are full
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop.one_step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.one_step()
    held, evictions = 1, []
    for step in range(1, steps):
        if held == room:
            evictions.append((step, eviction.weights.clone()))
            eviction.evict()
            evictions[-1] += (eviction.source.clone(), attn.suffix_lens.clone())
            held = budget
        graph.replay()
        held += 1
    loop.flush()
    torch.cuda.synchronize()
    return {"prompt_pass": prompt_pass, "qkv": (q, k, v), "weights": weights, "source": source, "kept": kept, "prefix_lens": prefix_lens,
            "loop": loop, "logits": logits, "evictions": evictions, "prompt_lens": prompt_lens, "samples_per_prompt": samples_per_prompt,
            "sinks": sinks, "recent": recent, "budget": budget, "room": room, "num_top": num_top}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=96)
    a = ap.parse_args()
    got = run(steps=a.steps)
    loop = got["loop"]
    print(f"room was made {len(got['evictions'])} times; a sample holds {loop.attn.suffix_lens[0]} of its {a.steps} tokens")
    for r in range(0, loop.tokens_steps.shape[1], 4):
        steps = [f"{t} ({p:.2f})" for t, p in zip(loop.tokens_steps[:8, r].tolist(), loop.logprobs_steps[:8, r].tolist())]
        print(f"sample {r}: {' '.join(steps)} ...")
