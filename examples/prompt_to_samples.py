"""From request lengths to sampled tokens, all on the device: the pages of a few prompts and of their samples, the
prompts' keys, values and attention, and a captured loop of decode steps whose logits are shaped by repetition and
frequency penalties, a bias and a grammar mask.

Keys, queries, values and logits are random (there are no weights here); everything else is what a server does.

    python examples/prompt_to_samples.py [--steps 32]
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


def run(prompt_lens=(700, 1203, 64), samples_per_prompt=4, steps=16, vocab=32000, seed=0, dev="cuda:0"):
    """Returns what a test needs: the prompt pass, the decode loop, the inputs of the logits' shaping."""
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)  # noqa: E731
    prompts, rows, tokens = len(prompt_lens), len(prompt_lens) * samples_per_prompt, sum(prompt_lens)

    # the cache, with its pages handed out in no particular order
    prompt_pages = sum(-(-n // PAGE) for n in prompt_lens)
    sample_pages = rows * -(-steps // PAGE)
    pool = (prompt_pages + sample_pages + 5, HKV, PAGE, HEAD_DIM)
    k_pool, v_pool = (torch.zeros(pool, dtype=torch.bfloat16, device=dev) for _ in range(2))
    free = torch.randperm(pool[0], generator=g, device=dev).to(torch.int32)

    # 1. pages for the prompts, then, from the rest of the list, for the samples' own tokens
    lens = _i32(prompt_lens, dev)
    prompt_tables = D.build_tables(lens, free, prompt_pages, tokens)
    sample_tables = D.build_tables(torch.full((rows,), steps, dtype=torch.int32, device=dev), free, sample_pages,
                                   free_begin=prompt_tables.free_end)

    # 2. the prompts: q, k and v as one projection leaves them, into the pages, and their attention
    qkv = normal(tokens, (HQ + 2 * HKV) * HEAD_DIM)
    q = qkv[:, : HQ * HEAD_DIM].unflatten(1, (HQ, HEAD_DIM))
    k = qkv[:, HQ * HEAD_DIM:(HQ + HKV) * HEAD_DIM].unflatten(1, (HKV, HEAD_DIM))
    v = qkv[:, (HQ + HKV) * HEAD_DIM:].unflatten(1, (HKV, HEAD_DIM))
    prompt_pass = D.DevicePrompts(prompt_tables, q, k, v, k_pool, v_pool, max(prompt_lens), max(prompt_lens))
    prompt_pass.run()

    # 3. which tokens each prompt holds
    prompt_tokens = torch.randint(0, vocab, (tokens,), generator=g, device=dev, dtype=torch.int32)
    words = -(-vocab // 32)
    prompt_bits = torch.empty((prompts, words), dtype=torch.int32, device=dev)
    B.mark_prompt_tokens(prompt_tokens, prompt_tables.packed_indptr, prompts, vocab, prompt_bits, words)

    # 4. decode: attention over the prompt's pages and the sample's own, greedy sampling of shaped logits
    desc = B.make_desc(dtype=B.SPD_BF16, num_q_heads=HQ, num_kv_heads=HKV, head_dim=HEAD_DIM, num_prompts=prompts, num_samples=rows,
                       max_samples_per_prompt=samples_per_prompt, page_size=PAGE)
    ws = torch.empty(B.shared_prefix_decode_attn_workspace_size(desc, max(prompt_lens), steps), dtype=torch.uint8, device=dev)
    sample_indptr = _i32([i * samples_per_prompt for i in range(prompts + 1)], dev)
    attn = D.DeviceAttn(desc, normal(rows, HQ, HEAD_DIM), k_pool, v_pool, prompt_tables.lens, prompt_tables.page_indptr,
                        prompt_tables.page_indices, sample_indptr, k_pool, v_pool,
                        torch.zeros(rows, dtype=torch.int32, device=dev), sample_tables.page_indptr, sample_tables.page_indices,
                        max(prompt_lens), steps, normal(rows, HQ, HEAD_DIM), torch.empty((rows, HQ), device=dev), ws)
    shaped = torch.empty((rows, vocab), device=dev)
    sampler = D.DeviceSampler(shaped, torch.zeros(rows, device=dev), torch.ones(rows, device=dev), torch.zeros(rows, device=dev),
                              torch.empty(rows, dtype=torch.int32, device=dev),
                              torch.empty(B.sample_tokens_workspace_size(rows, vocab), dtype=torch.uint8, device=dev))
    raw = normal(rows, vocab) * 3
    grammar = torch.full((1, words), -1, dtype=torch.int32, device=dev)
    grammar[0, : words // 2] = 0x55555555  # one state: even tokens only in the first half of the vocabulary
    row = torch.arange(rows, device=dev, dtype=torch.int32)
    shaping = dict(repetition=torch.full((rows,), 1.2, device=dev), frequency=torch.full((rows,), 0.7, device=dev),
                   presence=torch.full((rows,), 0.3, device=dev), prompt_bits=prompt_bits, prompt_of_row=row // samples_per_prompt,
                   bias_indptr=torch.arange(rows + 1, device=dev, dtype=torch.int32), bias_tokens=(row * 7 + 3) % vocab,
                   bias_values=torch.full((rows,), 2.5, device=dev), allowed_bits=grammar,
                   allowed_of_row=torch.where(row % 2 == 0, 0, -1).to(torch.int32))
    loop = D.DecodeLoop(attn, sampler, normal(steps, rows, HQ, HEAD_DIM), normal(steps, rows, HKV, HEAD_DIM),
                        normal(steps, rows, HKV, HEAD_DIM), torch.zeros((steps, rows), device=dev), end_token=-2,  # (a token that is never drawn)
                        raw_logits=raw, penalties=shaping)

    # one step as it is, the rest replayed from one captured step
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop.one_step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.one_step()
    for _ in range(steps - 1):
        graph.replay()
    loop.flush()
    torch.cuda.synchronize()
    return {"prompt_pass": prompt_pass, "prompt_tables": prompt_tables, "sample_tables": sample_tables, "loop": loop, "raw": raw,
            "shaping": shaping, "prompt_tokens": prompt_tokens, "prompt_lens": prompt_lens, "samples_per_prompt": samples_per_prompt,
            "free": free, "qkv": (q, k, v)}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    got = run(steps=a.steps)
    tokens = got["loop"].tokens_steps.t()
    for r in range(0, tokens.shape[0], 4):
        print(f"sample {r}: {tokens[r, :12].tolist()} ...")
