"""Performance cases of the operators between a request and its first token, and between logits and the sampler.

Five kinds of case, each a dict of plain values:

  prompt  attention of a batch of prompts' new tokens over everything before them (`prompt_attn`): packed
          prompts of different lengths, causal or not, fp32 or bf16, contiguous or paged KV, with or
          without tokens that are in the cache already
  tables  page tables, slot map and granted lengths from request lengths (`build_page_tables`)
  write   the prompts' keys and values into the pages of the cache (`write_prompt_kv`)
  mark    which tokens of the vocabulary occur in each prompt (`mark_prompt_tokens`)
  logits  repetition, frequency and presence penalties, biases and a grammar mask (`penalize_logits`)

Sizes are those of the library's configurations (`workloads.SPECS`) and of `perf/cases.py`, or generic.
With `own` false the operators run in their plain form, in torch operations of 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
PAGE = 16
INF = float("inf")


# ---- the cases ----------------------------------------------------------------------------------------

def _prompt(name, dtype, hq, hkv, d, prompts, new, past=(0, 0), page=0, causal=1, fused=0):
    return {"name": name, "kind": "prompt", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "prompts": prompts,
            "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "page": page, "causal": causal,
            "fused": fused}


def _tables(name, requests, new, past=(0, 0), free_percent=110):
    return {"name": name, "kind": "tables", "requests": requests, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
            "past_hi": past[1], "free_percent": free_percent}


def _write(name, dtype, hkv, d, prompts, tokens, fused=0):
    return {"name": name, "kind": "write", "dtype": dtype, "hkv": hkv, "d": d, "prompts": prompts, "new_lo": tokens[0],
            "new_hi": tokens[1], "fused": fused}


def _mark(name, prompts, tokens, vocab):
    return {"name": name, "kind": "mark", "prompts": prompts, "new_lo": tokens[0], "new_hi": tokens[1], "vocab": vocab}


def _logits(name, dtype, prompts, spp, vocab, prompt_tokens, generated, biases, grammars, by_step=1):
    return {"name": name, "kind": "logits", "dtype": dtype, "prompts": prompts, "spp": spp, "vocab": vocab,
            "prompt_tokens": prompt_tokens, "gen_lo": generated[0], "gen_hi": generated[1], "biases": biases,
            "grammars": grammars, "by_step": by_step}


def listed():
    return [
        # the smallest prompt (configuration 1): 256 tokens, fp32, all latency
        _prompt("prompt-f32-256", "f32", 4, 1, 64, 1, (256, 256)),
        # a model with 64-channel heads, three prompts of odd lengths, q, k and v slices of one projection
        _prompt("prompt-d64-ragged", "bf16", 32, 8, 64, 3, (500, 4001), fused=1),
        # four conversations that go on: a few dozen new tokens each over what the cache holds, paged
        _prompt("prompt-turn-paged", "bf16", 32, 8, 128, 4, (17, 96), past=(2048, 8192), page=PAGE),
        # one layer of a large model (64 query heads) over a whole 16k prompt (configuration 4): the largest
        _prompt("prompt-16k-g8", "bf16", 64, 8, 128, 1, (16384, 16384)),
        # the prompts of a serving batch (configuration 5) get their pages
        _tables("tables-prompts-8", 8, (1024, 16384)),
        # its 1024 samples in the middle of their generation grow by up to 16 tokens
        _tables("tables-samples-1024", 1024, (1, 16), past=(0, 2032)),
        # the smallest write (configuration 1)
        _write("write-f32-256", "f32", 1, 64, 1, (256, 256)),
        # one layer's keys and values of the serving batch's prompts
        _write("write-prompts-8", "bf16", 8, 128, 8, (1024, 16384)),
        # one prompt of the sampling job (configuration 3)
        _mark("mark-8k", 1, (8192, 8192), 128256),
        # the prompts of the serving batch
        _mark("mark-prompts-8", 8, (1024, 16384), 128256),
        # 64 completions of one prompt, up to 1024 generated tokens, a few biases, fp32 logits (configuration 3)
        _logits("logits-n64", "f32", 1, 64, 128256, 8192, (128, 1024), 32, 0),
        # the serving batch: 1024 rows of bf16 logits, half of them held to one of 16 grammar states
        _logits("logits-n1024-grammar", "bf16", 8, 128, 128256, 8704, (0, 2048), 8, 16),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _range(rng, lo, hi):
    a, b = _logint(rng, lo, hi), _logint(rng, lo, hi)
    return min(a, b), max(a, b)


def draw(rng):
    kind = rng.choices(["prompt", "tables", "write", "mark", "logits"], [5, 2, 2, 1, 3])[0]
    if kind == "prompt":
        while True:
            hkv = rng.choice([1, 2, 4, 8])
            past = (0, 0) if rng.random() < 0.6 else _range(rng, 16, 12000)
            page = PAGE if rng.random() < 0.5 else 0
            c = _prompt("", "bf16" if rng.random() < 0.75 else "f32", hkv * rng.choice([1, 2, 4, 8]), hkv,
                        rng.choice([64, 64, 80, 96, 128, 128, 128, 256]), _logint(rng, 1, 26), _range(rng, 1, 8192), past, page,
                        0 if rng.random() < 0.15 else 1, 1 if past == (0, 0) and not page and rng.random() < 0.5 else 0)
            w = work(c)
            scores = c["prompts"] * c["hq"] * c["new_hi"] * (c["new_hi"] + c["past_hi"])
            if scores <= 4e9 and w["flops"] <= (1.5e12 if c["dtype"] == "bf16" else 4e11) and w["bytes"] <= 4e8:
                break
    elif kind == "tables":
        while True:
            held = rng.random() < 0.5
            c = _tables("", _logint(rng, 1, 8192), _range(rng, 1, 64 if held else 16384), _range(rng, 1, 2048) if held else (0, 0),
                        rng.choice([100, 110, 150, 60]))
            if work(c)["bytes"] <= 4e6:
                break
    elif kind == "write":
        while True:
            c = _write("", rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 256]),
                       _logint(rng, 1, 32), _range(rng, 1, 16384), rng.choice([0, 1]))
            if work(c)["bytes"] <= 5e8:
                break
    elif kind == "mark":
        c = _mark("", _logint(rng, 1, 32), _range(rng, 1, 8704), rng.choice([1024, 32000, 50257, 128256]))
    else:
        while True:
            c = _logits("", rng.choice(["bf16", "f32"]), _logint(rng, 1, 8), _logint(rng, 1, 128),
                        rng.choice([1024, 32000, 50257, 128256]), _logint(rng, 1, 16384), _range(rng, 1, 2048),
                        rng.choice([0, 5, 40, 300]), rng.choice([0, 0, 1, 16]), rng.choice([0, 1]))
            if work(c)["bytes"] <= 7e8:
                break
    c.pop("name", None)
    return c


# ---- inputs ---------------------------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n lengths from lo to hi, both among them where n > 1: the same ones for every seed, so that the work is."""
    return [lo + (hi - lo) * i // (n - 1) for i in range(n)] if n > 1 else [(lo + hi) // 2]


def _shuffled(seed, which, lo, hi, n):
    lens = _spread(lo, hi, n)
    random.Random("%d %s" % (seed, which)).shuffle(lens)
    return lens


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _type(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _tokens(g, shape, vocab):
    """Token ids that crowd at the low end, as words of a text do."""
    return (vocab * torch.rand(shape, generator=g, device=DEV) ** 3).to(torch.int32).clamp_(max=vocab - 1)


def _rows(g, tokens, heads, d, dtype, parts, fused):
    """`parts` tensors [tokens, heads, d], of their own or (fused) slices of one [tokens, everything] tensor."""
    wide = torch.randn((tokens, sum(heads) * d), generator=g, device=DEV, dtype=_type(dtype))
    got, at = [], 0
    for i in range(parts):
        part = wide[:, at:at + heads[i] * d].unflatten(1, (heads[i], d))
        got.append(part if fused else part.contiguous())
        at += heads[i] * d
    return got


def _prepare_prompt(c, seed):
    g = _gen(seed)
    hq, hkv, d, n = c["hq"], c["hkv"], c["d"], c["prompts"]
    new = _shuffled(seed, "new", c["new_lo"], c["new_hi"], n)
    past = _shuffled(seed, "past", c["past_lo"], c["past_hi"], n)
    kv = [a + b for a, b in zip(new, past)]
    s = {"case": c, "new_starts": _ints(_starts(new)), "kv_lens": _ints(kv), "total": sum(new), "max_new": max(new),
         "max_kv": max(kv), "pages": None}
    if c["page"]:
        held = [-(-x // PAGE) for x in kv]
        s["kv_starts"] = _ints(_starts(held))
        s["pages"] = torch.randperm(sum(held), generator=g, device=DEV).to(torch.int32)
        s["q"], = _rows(g, sum(new), [hq], d, c["dtype"], 1, 0)
        pool = (sum(held), hkv, PAGE, d)
        s["k"] = torch.randn(pool, generator=g, device=DEV, dtype=_type(c["dtype"]))
        s["v"] = torch.randn(pool, generator=g, device=DEV, dtype=_type(c["dtype"]))
    elif c["fused"]:
        s["kv_starts"] = s["new_starts"]
        s["q"], s["k"], s["v"] = _rows(g, sum(new), [hq, hkv, hkv], d, c["dtype"], 3, 1)
    else:
        s["kv_starts"] = _ints(_starts(kv))
        s["q"], = _rows(g, sum(new), [hq], d, c["dtype"], 1, 0)
        s["k"], s["v"] = _rows(g, sum(kv), [hkv, hkv], d, c["dtype"], 2, 0)
    s["q"].mul_(2.0)  # scores of standard deviation 2: some tokens count for far more than others
    s["out"] = torch.empty((sum(new), hq, d), dtype=_type(c["dtype"]), device=DEV)
    s["lse"] = torch.empty((sum(new), hq), dtype=torch.float32, device=DEV)
    return s


def _prepare_tables(c, seed):
    g, n = _gen(seed), c["requests"]
    new = _shuffled(seed, "new", c["new_lo"], c["new_hi"], n)
    past = _shuffled(seed, "past", c["past_lo"], c["past_hi"], n)
    held = [-(-x // PAGE) for x in past]
    need = sum(-(-(a + b) // PAGE) for a, b in zip(new, past)) - sum(held)
    free = max(1, need * c["free_percent"] // 100)
    perm = torch.randperm(sum(held) + free, generator=g, device=DEV).to(torch.int32)
    s = {"case": c, "lens": _ints([a + b for a, b in zip(new, past)]), "held_lens": None, "held_starts": None,
         "held_pages": None, "free": perm[sum(held):].clone(), "max_pages": (sum(new) + sum(past)) // PAGE + n, "max_tokens": sum(new)}
    if c["past_hi"]:
        s.update(held_lens=_ints(past), held_starts=_ints(_starts(held)), held_pages=perm[:sum(held)].clone())
    empty = lambda n, t=torch.int32: torch.empty(n, dtype=t, device=DEV)  # noqa: E731
    s["out"] = {"page_indptr": empty(n + 1), "page_indices": empty(s["max_pages"]), "lens": empty(n), "new_indptr": empty(n + 1),
                "slots": empty(s["max_tokens"], torch.int64), "free_end": empty(1)}
    return s


def _prepare_write(c, seed):
    g = _gen(seed)
    lens = _shuffled(seed, "new", c["new_lo"], c["new_hi"], c["prompts"])
    held = [-(-x // PAGE) for x in lens]
    pages = torch.randperm(sum(held), generator=g, device=DEV)
    first = _starts(held)
    slots = torch.cat([(pages[first[i]:first[i + 1], None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(-1)[:n]
                       for i, n in enumerate(lens)])
    # a fused projection holds the queries too, four heads for each of the keys
    heads = [c["hkv"], c["hkv"]] + ([4 * c["hkv"]] if c["fused"] else [])
    k, v = _rows(g, sum(lens), heads, c["d"], c["dtype"], 2, c["fused"])
    pool = (sum(held), c["hkv"], PAGE, c["d"])
    return {"case": c, "k": k, "v": v, "slots": slots, "k_pool": torch.zeros(pool, dtype=k.dtype, device=DEV),
            "v_pool": torch.zeros(pool, dtype=k.dtype, device=DEV)}


def _prepare_mark(c, seed):
    lens = _shuffled(seed, "new", c["new_lo"], c["new_hi"], c["prompts"])
    words = -(-c["vocab"] // 32)
    return {"case": c, "tokens": _tokens(_gen(seed), (sum(lens),), c["vocab"]), "starts": _ints(_starts(lens)),
            "bits": torch.empty((c["prompts"], words), dtype=torch.int32, device=DEV)}


def _prepare_logits(c, seed):
    g, vocab, rows = _gen(seed), c["vocab"], c["prompts"] * c["spp"]
    words, most = -(-vocab // 32), c["gen_hi"]
    x = torch.randn((rows, vocab), generator=g, device=DEV) * 3.0
    s = {"case": c, "logits": x.to(_type(c["dtype"])), "out": torch.empty((rows, vocab), dtype=torch.float32, device=DEV)}
    marks = torch.zeros((c["prompts"], words * 32), dtype=torch.int64, device=DEV)
    marks.scatter_(1, _tokens(g, (c["prompts"], c["prompt_tokens"]), vocab).long(), 1)
    s["prompt_bits"] = _packed(marks)
    s["prompt_of_row"] = torch.arange(rows, device=DEV, dtype=torch.int32) // c["spp"]
    tokens = _tokens(g, (rows, most), vocab)
    s["tokens"] = tokens.t().contiguous().t() if c["by_step"] else tokens  # a loop's record is [steps, rows]
    s["token_lens"] = _ints(_shuffled(seed, "gen", c["gen_lo"], c["gen_hi"], rows))
    s["repetition"] = 1.0 + 0.3 * torch.rand(rows, generator=g, device=DEV)
    s["frequency"] = 0.5 * torch.rand(rows, generator=g, device=DEV)
    s["presence"] = 0.5 * torch.rand(rows, generator=g, device=DEV)
    s["bias_starts"] = s["bias_tokens"] = s["bias_values"] = s["allowed_bits"] = s["allowed_of_row"] = None
    if c["biases"]:
        # up to `biases` different tokens a row, one from each stretch of the vocabulary
        counts = _shuffled(seed, "bias", 0, c["biases"], rows)
        part = vocab // c["biases"]
        at = torch.arange(c["biases"], device=DEV) * part + torch.randint(0, part, (rows, c["biases"]), generator=g, device=DEV)
        keep = torch.arange(c["biases"], device=DEV) < _ints(counts)[:, None]
        s["bias_starts"] = _ints(_starts(counts))
        s["bias_tokens"] = at[keep].to(torch.int32)
        s["bias_values"] = 4.0 * torch.randn(int(sum(counts)), generator=g, device=DEV)
    if c["grammars"]:
        # states that allow a few tokens, or most of them; every other row is free
        share = 0.002 + 0.97 * (torch.arange(c["grammars"], device=DEV) % 2)[:, None]
        s["allowed_bits"] = _packed((torch.rand((c["grammars"], words * 32), generator=g, device=DEV) < share).long())
        row = torch.arange(rows, device=DEV, dtype=torch.int32)
        s["allowed_of_row"] = torch.where(row % 2 == 0, row // 2 % c["grammars"], -1)
    return s


def _packed(marks):
    """[rows, 32 w] zeros and ones as [rows, w] words of 32 bits."""
    words = (marks.unflatten(1, (-1, 32)) << torch.arange(32, device=marks.device)).sum(-1)
    return words.to(torch.int32)


def prepare(case, seed):
    return {"prompt": _prepare_prompt, "tables": _prepare_tables, "write": _prepare_write, "mark": _prepare_mark,
            "logits": _prepare_logits}[case["kind"]](case, seed)


# ---- the framework's calls ----------------------------------------------------------------------------------

def _handle(s):
    """What a program sets up once for such a call: the description and the workspace."""
    from paper_2502_02534_amd import binding as B
    c = s["case"]
    if c["kind"] in ("prompt", "write"):
        row = lambda name: s[name].stride(0) if c["fused"] and name in s else 0  # noqa: E731
        desc = B.make_prompt_desc(dtype=B.SPD_F32 if c["dtype"] == "f32" else B.SPD_BF16, num_q_heads=c.get("hq", c["hkv"]),
                                  num_kv_heads=c["hkv"], head_dim=c["d"], num_prompts=c["prompts"],
                                  page_size=PAGE if c["kind"] == "write" else c["page"], causal=c.get("causal", 1),
                                  q_stride=row("q"), kv_stride=row("k"))
        size = B.prompt_attn_workspace_size(desc, s["total"], s["max_new"], s["max_kv"]) if c["kind"] == "prompt" else 0
        return B, desc, torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)
    if c["kind"] == "tables":
        return B, None, torch.empty(max(B.build_page_tables_workspace_size(c["requests"]), 256), dtype=torch.uint8, device=DEV)
    if c["kind"] == "logits":
        return B, B.make_penalties(repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                                   prompt_bits=s["prompt_bits"], prompt_of_row=s["prompt_of_row"], tokens=s["tokens"],
                                   token_lens=s["token_lens"], bias_indptr=s["bias_starts"], bias_tokens=s["bias_tokens"],
                                   bias_values=s["bias_values"], allowed_bits=s["allowed_bits"],
                                   allowed_of_row=s["allowed_of_row"]), None
    return B, None, None


def _run_own(s):
    c = s["case"]
    if "handle" not in s:
        s["handle"] = _handle(s)
    B, desc, ws = s["handle"]
    if c["kind"] == "prompt":
        B.prompt_attn(desc, s["q"], s["k"], s["v"], s["new_starts"], s["kv_lens"], s["kv_starts"], s["pages"], s["total"],
                      s["max_new"], s["max_kv"], s["out"], s["lse"], ws)
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "tables":
        o = s["out"]
        B.build_page_tables(c["requests"], PAGE, s["lens"], s["held_lens"], s["held_starts"], s["held_pages"], s["free"],
                            s["free"].numel(), None, s["max_pages"], s["max_tokens"], o["page_indptr"], o["page_indices"],
                            o["lens"], o["new_indptr"], o["slots"], o["free_end"], ws)
        return o
    if c["kind"] == "write":
        B.write_prompt_kv(desc, s["k"], s["v"], s["slots"], s["slots"].numel(), s["k_pool"].shape[0], s["k_pool"], s["v_pool"])
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if c["kind"] == "mark":
        B.mark_prompt_tokens(s["tokens"], s["starts"], c["prompts"], c["vocab"], s["bits"], s["bits"].stride(0))
        return s["bits"]
    rows, vocab = s["logits"].shape
    B.penalize_logits(s["logits"], B.SPD_F32 if c["dtype"] == "f32" else B.SPD_BF16, rows, vocab, s["logits"].stride(0), desc,
                      s["out"], s["out"].stride(0))
    return s["out"]


# ---- the plain forms ----------------------------------------------------------------------------------------

def _which(starts, total):
    """For each of `total` packed places, the index of the range of `starts` that it lies in, and its place there."""
    t = torch.arange(total, device=DEV, dtype=torch.int32)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp_(max=starts.numel() - 2)
    return b, t - starts[b]


def _plain_prompt(s):
    c = s["case"]
    hq, hkv, d, n = c["hq"], c["hkv"], c["d"], c["prompts"]
    starts, kv_lens, mq, mk = s["new_starts"], s["kv_lens"], s["max_new"], s["max_kv"]
    new = starts[1:] - starts[:-1]
    i = torch.arange(mq, device=DEV)
    q = s["q"].float()[(starts[:-1, None] + i).clamp(max=s["total"] - 1)]                    # [n, mq, hq, d]
    q = q.unflatten(2, (hkv, -1)).permute(0, 2, 1, 3, 4).reshape(n, hkv, mq * (hq // hkv), d)
    t = torch.arange(mk, device=DEV)
    if c["page"]:
        page = s["pages"][(s["kv_starts"][:-1, None] + t // PAGE).clamp(max=s["pages"].numel() - 1)]
        k, v = s["k"][page, :, t % PAGE].float(), s["v"][page, :, t % PAGE].float()            # [n, mk, hkv, d]
    else:
        at = (s["kv_starts"][:-1, None] + t).clamp(max=s["k"].shape[0] - 1)
        k, v = s["k"].float()[at], s["v"].float()[at]
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(d))
    seen = (t < kv_lens[:, None])[:, None, :].expand(n, mq, mk)
    if c["causal"]:
        seen = seen & (t <= (kv_lens - new)[:, None, None] + i[:, None])
    x.unflatten(2, (mq, -1)).masked_fill_(~seen[:, None, :, None, :], -INF)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -INF, 0.0, m)
    x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v.transpose(1, 2).contiguous()) / torch.where(l == 0, 1.0, l)
    lse = (m + torch.log(l)).squeeze(-1).unflatten(2, (mq, -1)).permute(0, 2, 1, 3).reshape(n, mq, hq)
    o = o.unflatten(2, (mq, -1)).permute(0, 2, 1, 3, 4).reshape(n, mq, hq, d)
    b, at = _which(starts, s["total"])
    return {"out": o[b, at].to(s["q"].dtype), "lse": lse[b, at]}


def _plain_tables(s):
    o, lens = s["out"], s["lens"]
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    sums = lambda x: torch.cat([zero, torch.cumsum(x, 0, dtype=torch.int32)])  # noqa: E731
    if s["held_lens"] is None:
        held_lens, held, held_starts = torch.zeros_like(lens), torch.zeros_like(lens), sums(torch.zeros_like(lens))
        held_pages = zero
    else:
        held_lens, held_starts, held_pages = s["held_lens"], s["held_starts"], s["held_pages"]
        held = held_starts[1:] - held_starts[:-1]
    want = torch.maximum(lens, held_lens)
    need = ((want + PAGE - 1) // PAGE - held).clamp(min=0)
    granted = (need == 0) | (torch.cumsum(need, 0) <= s["free"].numel())
    taken = torch.where(granted, need, 0)
    free_starts, page_indptr = sums(taken), sums(held + taken)
    lens_out = torch.where(granted, want, held_lens)
    new_indptr = sums(lens_out - held_lens)

    def page(b, p):
        old = held_pages[(held_starts[b] + p).clamp(min=0, max=held_pages.numel() - 1)]
        fresh = s["free"][(free_starts[b] + p - held[b]).clamp(min=0, max=s["free"].numel() - 1)]
        return torch.where(p < held[b], old, fresh)

    b, p = _which(page_indptr, s["max_pages"])
    pages = torch.where(torch.arange(s["max_pages"], device=DEV) < page_indptr[-1], page(b, p), -1)
    b, at = _which(new_indptr, s["max_tokens"])
    at = at + held_lens[b]
    slots = torch.where(torch.arange(s["max_tokens"], device=DEV) < new_indptr[-1], page(b, at // PAGE).long() * PAGE + at % PAGE, -1)
    return {"page_indptr": page_indptr, "page_indices": pages, "lens": lens_out, "new_indptr": new_indptr, "slots": slots,
            "free_end": free_starts[-1:]}


def _plain_write(s):
    page, at = s["slots"] // PAGE, s["slots"] % PAGE
    s["k_pool"][page, :, at] = s["k"]
    s["v_pool"][page, :, at] = s["v"]
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_mark(s):
    words = s["bits"].shape[1]
    b, _ = _which(s["starts"], s["tokens"].numel())
    marks = torch.zeros((s["case"]["prompts"], words * 32), dtype=torch.int64, device=DEV)
    marks[b, s["tokens"].long()] = 1
    return _packed(marks)


def _unpacked(words, vocab):
    return ((words[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1).bool().flatten(1)[:, :vocab]


def _plain_logits(s):
    x = s["logits"].float()
    rows, vocab = x.shape
    t = torch.arange(s["tokens"].shape[1], device=DEV)
    counts = torch.zeros_like(x).scatter_add_(1, s["tokens"].long(), (t < s["token_lens"][:, None]).float())
    seen = (counts > 0) | _unpacked(s["prompt_bits"], vocab)[s["prompt_of_row"]]
    rho = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
    x = x - s["frequency"][:, None] * counts - s["presence"][:, None] * (counts > 0)
    if s["bias_tokens"] is not None:
        r, _ = _which(s["bias_starts"], s["bias_tokens"].numel())
        x.view(-1).scatter_add_(0, r * vocab + s["bias_tokens"], s["bias_values"])
    if s["allowed_bits"] is not None:
        allowed = _unpacked(s["allowed_bits"], vocab)[s["allowed_of_row"].clamp(min=0)]
        x.masked_fill_(~(allowed | (s["allowed_of_row"] < 0)[:, None]), -INF)
    return x


def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "tables": _plain_tables, "write": _plain_write, "mark": _plain_mark,
            "logits": _plain_logits}[state["case"]["kind"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(case):
    c, e = case, 4 if case.get("dtype") == "f32" else 2
    if c["kind"] == "prompt":
        # prompts' new and cached lengths are paired at random: the sums of products go by the means
        new, past = (_spread(c[w + "_lo"], c[w + "_hi"], c["prompts"]) for w in ("new", "past"))
        mean_past = sum(past) / len(past)
        pairs = sum(x * mean_past + (x * (x + 1) / 2 if c["causal"] else x * x) for x in new)
        byte = (sum(new) + sum(past)) * 2 * c["hkv"] * c["d"] * e + sum(new) * c["hq"] * (2 * c["d"] * e + 4)
        return {"bytes": byte, "flops": 4 * c["d"] * c["hq"] * pairs}
    if c["kind"] == "tables":
        new, past = (_spread(c[w + "_lo"], c[w + "_hi"], c["requests"]) for w in ("new", "past"))
        held = sum(-(-x // PAGE) for x in past)
        pages = (sum(new) + sum(past)) // PAGE + c["requests"] // 2
        return {"bytes": 4 * c["requests"] * (6 if held else 4) + 8 * pages + 8 * sum(new), "flops": 0}
    if c["kind"] == "write":
        return {"bytes": sum(_spread(c["new_lo"], c["new_hi"], c["prompts"])) * (4 * c["hkv"] * c["d"] * e + 8), "flops": 0}
    if c["kind"] == "mark":
        return {"bytes": 4 * sum(_spread(c["new_lo"], c["new_hi"], c["prompts"])) + c["prompts"] * -(-c["vocab"] // 8), "flops": 0}
    rows = c["prompts"] * c["spp"]
    lists = sum(_spread(c["gen_lo"], c["gen_hi"], rows)) * 4 + sum(_spread(0, c["biases"], rows)) * 8
    bits = (c["prompts"] + c["grammars"]) * -(-c["vocab"] // 8)
    return {"bytes": rows * (c["vocab"] * (e + 4) + 28) + lists + bits, "flops": 0}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _exact_prompt(c, s):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    out = torch.empty((s["total"], hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((s["total"], hq), dtype=torch.float64, device=DEV)
    starts, kv_starts, lens = s["new_starts"].tolist(), s["kv_starts"].tolist(), s["kv_lens"].tolist()
    for b in range(c["prompts"]):
        q0, n, length = starts[b], starts[b + 1] - starts[b], lens[b]
        for j in range(hkv):
            if c["page"]:
                ids = s["pages"][kv_starts[b]:kv_starts[b + 1]].long()
                k, v = (s[w][ids, j].reshape(-1, d)[:length].double() for w in "kv")
            else:
                k, v = (s[w][kv_starts[b]:kv_starts[b] + length, j].double() for w in "kv")
            for first in range(0, n, 2048):
                last = min(n, first + 2048)
                limit = length - n + torch.arange(first, last, device=DEV) if c["causal"] else None
                for h in range(j * g, j * g + g):
                    scores = s["q"][q0 + first:q0 + last, h].double() @ k.T / d ** 0.5
                    if limit is not None:
                        scores[torch.arange(length, device=DEV)[None, :] > limit[:, None]] = -INF
                    total = torch.logsumexp(scores, 1)
                    lse[q0 + first:q0 + last, h] = total
                    out[q0 + first:q0 + last, h] = torch.exp(scores - total[:, None]) @ v
    return {"out": out, "lse": lse}


def _exact_logits(c, s):
    rows, vocab = s["logits"].shape
    out = s["logits"].double()
    bit = torch.arange(vocab, device=DEV)
    for r in range(rows):
        mine = s["tokens"][r, :int(s["token_lens"][r])].long()
        count = torch.bincount(mine, minlength=vocab).double()
        words = s["prompt_bits"][int(s["prompt_of_row"][r])]
        seen = (count > 0) | ((words[bit // 32] >> (bit % 32).int()) % 2 != 0)
        x, rho = out[r], s["repetition"][r].double()
        x[seen] = torch.where(x[seen] > 0, x[seen] / rho, x[seen] * rho)
        x -= s["frequency"][r].double() * count
        x[count > 0] -= s["presence"][r].double()
        if s["bias_tokens"] is not None:
            a, b = s["bias_starts"][r], s["bias_starts"][r + 1]
            x[s["bias_tokens"][a:b].long()] += s["bias_values"][a:b].double()
        if s["allowed_bits"] is not None and int(s["allowed_of_row"][r]) >= 0:
            words = s["allowed_bits"][int(s["allowed_of_row"][r])]
            x[(words[bit // 32] >> (bit % 32).int()) % 2 == 0] = -INF
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "prompt":
        return _exact_prompt(case, s)
    if case["kind"] == "logits":
        return _exact_logits(case, s)
    if case["kind"] == "write":
        # a copy has one right value: that of the row whose slot it is
        got = {}
        for name in "kv":
            rows = torch.zeros((s["k_pool"].shape[0] * PAGE, case["hkv"], case["d"]), dtype=torch.float64, device=DEV)
            rows.index_copy_(0, s["slots"], s[name].double())
            got[name + "_pool"] = rows.unflatten(0, (-1, PAGE)).transpose(1, 2).contiguous()
        return got
    return None  # whole numbers
