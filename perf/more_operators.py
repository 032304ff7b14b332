"""Performance cases of what a decode step's two softmaxes say: which cached tokens the attention looked at, and how
probable the tokens are.

Four kinds of case, each a dict of plain values:

  logprobs  log probability and rank of a given token, entropy and the most probable tokens of every row of logits
            (`token_logprobs`)
  weights   attention weight that every cached token got, summed over queries and the heads of its KV head
            (`accumulate_kv_weights`): samples over a shared prompt, one query over a sample's own tokens, whole
            prompts, or their last tokens only
  select    which tokens of a cache stay, by accumulated weight (`select_kv_tokens`)
  compact   the keys, values and weights of the tokens that stay, moved together (`compact_kv`)

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

def _logprobs(name, dtype, rows, vocab, top, hot=0, pad=0):
    """`hot`: rows at temperatures of their own; `pad`: elements between the rows."""
    return {"name": name, "kind": "logprobs", "dtype": dtype, "rows": rows, "vocab": vocab, "top": top, "hot": hot, "pad": pad}


def _weights(name, dtype, hq, hkv, d, seqs, new, past, page=0, causal=0, elsewhere=0, sums=1):
    """Sequences of `past` tokens (and, causal, the `new` ones) under `new` queries each, whose softmax runs over about
    `elsewhere` more tokens that this cache does not hold; `sums`: added to what there is."""
    return {"name": name, "kind": "weights", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "seqs": seqs, "new_lo": new[0],
            "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "page": page, "causal": causal, "elsewhere": elsewhere,
            "sums": sums}


def _select(name, seqs, heads, lens, budget=0, percent=0, sinks=4, recent=64):
    """A budget of so many tokens, or of `percent` of each sequence's."""
    return {"name": name, "kind": "select", "seqs": seqs, "heads": heads, "len_lo": lens[0], "len_hi": lens[1], "budget": budget,
            "percent": percent, "sinks": sinks, "recent": recent}


def _compact(name, dtype, hkv, d, seqs, lens, budget=0, percent=0, in_place=0, page=PAGE):
    return {"name": name, "kind": "compact", "dtype": dtype, "hkv": hkv, "d": d, "seqs": seqs, "len_lo": lens[0], "len_hi": lens[1],
            "budget": budget, "percent": percent, "in_place": in_place, "page": page}


def listed():
    return [
        # the smallest call (configuration 1): four rows, all latency
        _logprobs("logprobs-f32-4", "f32", 4, 1024, 5),
        # the sampling job (configuration 3): 64 completions a step, 20 alternatives each
        _logprobs("logprobs-n64-top20", "f32", 64, 128256, 20),
        # the serving batch (configuration 5): bf16 logits, each prompt at its own temperature
        _logprobs("logprobs-n1024", "bf16", 1024, 128256, 5, hot=1),
        # a prompt's own tokens scored, one row each, a vocabulary of odd size
        _logprobs("logprobs-prompt-odd", "bf16", 2000, 50257, 0),
        # the smallest cache (configuration 1): four samples over one prompt
        _weights("weights-f32-256", "f32", 4, 1, 64, 1, (4, 4), (256, 256), elsewhere=32),
        # the sampling job: 64 samples over the prompt that they share
        _weights("weights-shared-n64", "bf16", 32, 8, 128, 1, (64, 64), (8192, 8192), elsewhere=576),
        # the serving batch: 1024 samples over their own tokens, paged
        _weights("weights-own-n1024", "bf16", 32, 8, 128, 1024, (1, 1), (0, 2048), page=PAGE, elsewhere=8704),
        # one layer of a large model over a whole 16k prompt (configuration 4): the largest
        _weights("weights-prompt-16k", "bf16", 64, 8, 128, 1, (16384, 16384), (0, 0), causal=1, sums=0),
        # the serving batch's samples down to half of what they may hold
        _select("select-n1024", 1024, 8, (0, 2048), budget=1024),
        # a long prompt down to an eighth
        _select("select-prompt-16k", 1, 8, (16384, 16384), budget=2048),
        # the serving batch's samples in their own pages
        _compact("compact-n1024", "bf16", 8, 128, 1024, (0, 2048), budget=1024, in_place=1),
        # its prompts down to a quarter, into other pages (their own may be shared)
        _compact("compact-prompts-8", "bf16", 8, 128, 8, (1024, 16384), percent=25),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _range(rng, lo, hi):
    a, b = _logint(rng, lo, hi), _logint(rng, lo, hi)
    return min(a, b), max(a, b)


def _draw_weights(rng):
    while True:
        hkv = rng.choice([1, 2, 4, 8])
        use = rng.choice(["shared", "own", "prompt", "window"])
        seqs = _logint(rng, 1, 1024) if use == "own" else _logint(rng, 1, 16)
        new = {"shared": _range(rng, 2, 256), "own": (1, 1), "prompt": _range(rng, 1, 8192), "window": _range(rng, 1, 96)}[use]
        past = {"shared": _range(rng, 16, 16384), "own": (0, _logint(rng, 1, 2048)), "prompt": (0, 0),
                "window": _range(rng, 16, 16384)}[use]
        c = _weights("", "bf16" if rng.random() < 0.75 else "f32", hkv * rng.choice([1, 2, 4, 8]), hkv,
                     rng.choice([64, 64, 80, 96, 128, 128, 128, 256]), seqs, new, past, PAGE if rng.random() < 0.5 else 0,
                     1 if use in ("prompt", "window") else 0, rng.choice([0, 500, 8704]) if use in ("shared", "own") else 0,
                     rng.choice([0, 1]))
        w = work(c)
        scores = c["seqs"] * c["hq"] * c["new_hi"] * (c["past_hi"] + (c["new_hi"] if c["causal"] else 0))
        if scores <= 4e9 and w["flops"] <= (1.0e12 if c["dtype"] == "bf16" else 1.2e11) and w["bytes"] <= 2.2e9:
            return c


def _draw_lens(rng):
    """Sequences, their lengths, and a budget or a share."""
    lens = _range(rng, 1, 16384)
    if rng.random() < 0.5:
        return _logint(rng, 1, 1024), lens, _logint(rng, 1, 8192), 0
    return _logint(rng, 1, 1024), lens, 0, rng.choice([10, 25, 50, 90])


def draw(rng):
    kind = rng.choices(["logprobs", "weights", "select", "compact"], [4, 5, 3, 3])[0]
    while True:
        if kind == "logprobs":
            c = _logprobs("", rng.choice(["bf16", "f32"]), _logint(rng, 1, 4096), rng.choice([1024, 32000, 50257, 128256]),
                          rng.choice([0, 1, 5, 20, 64]), rng.choice([0, 1]), rng.choice([0, 0, 8, 63]))
            fits = work(c)["bytes"] <= 2.7e8
        elif kind == "weights":
            c, fits = _draw_weights(rng), True
        elif kind == "select":
            seqs, lens, budget, percent = _draw_lens(rng)
            c = _select("", seqs, rng.choice([1, 2, 4, 8]), lens, budget, percent, rng.choice([0, 4, 16]), rng.choice([0, 1, 64, 128]))
            fits = c["seqs"] * c["heads"] * c["len_hi"] <= 1.7e7
        else:
            seqs, lens, budget, percent = _draw_lens(rng)
            c = _compact("", rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 256]), seqs, lens,
                         budget, percent, rng.choice([0, 1]), rng.choice([PAGE, PAGE, 0]))
            fits = c["seqs"] * c["hkv"] * c["d"] * c["len_hi"] * (4 if c["dtype"] == "f32" else 2) <= 4.3e9
        if fits:
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


def _cache(g, lens, hkv, d, dtype, page, order=None):
    """Keys or values of sequences of these lengths, with their table: starts and (paged) pages in no particular order."""
    if page:
        held = [-(-x // PAGE) for x in lens]
        if order is None:
            order = torch.randperm(max(1, sum(held)), generator=g, device=DEV).to(torch.int32)
        return _ints(_starts(held)), order, (max(1, sum(held)), hkv, PAGE, d)
    return _ints(_starts(lens)), None, (max(1, sum(lens)), hkv, d)


def _prepare_logprobs(c, seed):
    g, rows, vocab, wide = _gen(seed), c["rows"], c["vocab"], c["vocab"] + c["pad"]
    x = torch.randn((rows, wide), generator=g, device=DEV) * 3.0
    # some tokens stand out of every row
    at = torch.randint(0, vocab, (rows, 50), generator=g, device=DEV)
    x.scatter_add_(1, at, torch.full_like(at, 8.0, dtype=torch.float32) * torch.rand(at.shape, generator=g, device=DEV))
    x = x.to(_type(c["dtype"]))[:, :vocab]
    t = 0.2 + torch.rand(rows, generator=g, device=DEV) if c["hot"] else None
    # the given tokens: drawn from the rows' own probabilities
    noise = -torch.log(-torch.log(torch.rand((rows, vocab), generator=g, device=DEV).clamp_(1e-20, 1 - 1e-7)))
    tokens = (x.float() / (t[:, None] if c["hot"] else 1.0) + noise).argmax(1).to(torch.int32)
    empty = lambda *n, t=torch.float32: torch.empty(n, dtype=t, device=DEV)  # noqa: E731
    out = {"logprobs": empty(rows), "ranks": empty(rows, t=torch.int32), "entropy": empty(rows), "lse": empty(rows)}
    if c["top"]:
        out.update(top_tokens=empty(rows, c["top"], t=torch.int32), top_logprobs=empty(rows, c["top"]))
    return {"case": c, "logits": x, "temperature": t, "tokens": tokens, "out": out}


def _prepare_weights(c, seed):
    g, n, hq, hkv, d = _gen(seed), c["seqs"], c["hq"], c["hkv"], c["d"]
    new = _shuffled(seed, "new", c["new_lo"], c["new_hi"], n)
    past = _shuffled(seed, "past", c["past_lo"], c["past_hi"], n)
    kv = [p + (q if c["causal"] else 0) for p, q in zip(past, new)]
    s = {"case": c, "new_starts": _ints(_starts(new)), "kv_lens": _ints(kv), "total": sum(new), "max_new": max(new),
         "max_kv": max(1, c["past_hi"] + (c["new_hi"] if c["causal"] else 0))}
    s["kv_starts"], s["pages"], pool = _cache(g, kv, hkv, d, c["dtype"], c["page"])
    s["k"] = torch.randn(pool, generator=g, device=DEV, dtype=_type(c["dtype"]))
    # scores of standard deviation 2: some tokens count for far more than others
    s["q"] = torch.randn((sum(new), hq, d), generator=g, device=DEV, dtype=_type(c["dtype"])) * 2.0
    x, seen = _scores(s)
    x.masked_fill_(~seen, -INF)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -INF, 0.0, m)
    lse = m[..., 0] + torch.log(x.sub_(m).exp_().sum(-1))
    del x, seen
    if c["elsewhere"]:
        lse = torch.logaddexp(lse, math.log(c["elsewhere"]) + 2.0 + 0.1 * torch.randn(lse.shape, generator=g, device=DEV))
    b, at = _which(s["new_starts"], s["total"])
    s["lse"] = lse.unflatten(2, (s["max_new"], -1)).permute(0, 2, 1, 3).reshape(n, s["max_new"], hq)[b, at].contiguous()
    shape = (n, hkv, s["max_kv"])
    s["weights"] = torch.rand(shape, generator=g, device=DEV) ** 4 if c["sums"] else None
    s["out"] = torch.zeros(shape, device=DEV)
    return s


def _budgets(c, lens):
    return [c["budget"] if c["budget"] else max(1, n * c["percent"] // 100) for n in lens]


def _prepare_select(c, seed):
    g, n, heads = _gen(seed), c["seqs"], c["heads"]
    lens = _shuffled(seed, "len", c["len_lo"], c["len_hi"], n)
    budgets = _budgets(c, lens)
    most = max(1, max(min(a, b) for a, b in zip(lens, budgets)))
    # accumulated weights: a few tokens have most of it
    weights = torch.exp(2.0 * torch.randn((n, heads, max(lens)), generator=g, device=DEV))
    return {"case": c, "weights": weights, "lens": _ints(lens), "budgets": _ints(budgets), "max_len": max(lens), "max_new": most,
            "out": {"source": torch.full((n, heads, most), -1, dtype=torch.int32, device=DEV),
                    "new_lens": torch.empty(n, dtype=torch.int32, device=DEV)}}


def _prepare_compact(c, seed):
    g, n, hkv, d, dtype = _gen(seed), c["seqs"], c["hkv"], c["d"], _type(c["dtype"])
    lens = _shuffled(seed, "len", c["len_lo"], c["len_hi"], n)
    budgets = _budgets(c, lens)
    new = [min(a, b) for a, b in zip(lens, budgets)]
    most = max(1, max(new))
    s = {"case": c, "new_lens": _ints(new), "max_new": most}
    # tokens that stay, at random; the ones from behind fill the gaps, so that a pass can be repeated in place
    s["source"] = torch.full((n, hkv, most), -1, dtype=torch.int32, device=DEV)
    weights = torch.rand((n, hkv, max(lens)), generator=g, device=DEV)
    s["source"], _ = _plain_source(weights, _ints(lens), _ints(budgets), 0, 0, s["source"])
    s["starts"], s["pages"], pool = _cache(g, lens, hkv, d, c["dtype"], c["page"])
    s["k"], s["v"] = (torch.randn(pool, generator=g, device=DEV, dtype=dtype) for _ in range(2))
    s["weights"], s["weights_out"] = weights, torch.empty((n, hkv, max(lens)), device=DEV)
    s["lens"] = torch.empty(n, dtype=torch.int32, device=DEV)
    if c["in_place"]:
        s.update(out_starts=s["starts"], out_pages=s["pages"], k_out=s["k"], v_out=s["v"])
    else:
        s["out_starts"], s["out_pages"], pool = _cache(g, new, hkv, d, c["dtype"], c["page"])
        s["k_out"], s["v_out"] = (torch.zeros(pool, dtype=dtype, device=DEV) for _ in range(2))
    return s


def prepare(case, seed):
    return {"logprobs": _prepare_logprobs, "weights": _prepare_weights, "select": _prepare_select,
            "compact": _prepare_compact}[case["kind"]](case, seed)


# ---- the framework's calls ----------------------------------------------------------------------------------

def _handle(s):
    """What a program sets up once for such a call: the description and the workspace."""
    from paper_2502_02534_amd import binding as B
    c, desc, size = s["case"], None, 0
    if c["kind"] in ("weights", "compact"):
        desc = B.make_prompt_desc(dtype=B.SPD_F32 if c["dtype"] == "f32" else B.SPD_BF16, num_q_heads=c.get("hq", c["hkv"]),
                                  num_kv_heads=c["hkv"], head_dim=c["d"], num_prompts=c["seqs"], page_size=c["page"],
                                  causal=bool(c.get("causal", 0)))
    if c["kind"] == "weights":
        size = B.accumulate_kv_weights_workspace_size(desc, s["total"], s["max_new"], s["max_kv"])
    elif c["kind"] == "logprobs":
        size = B.token_logprobs_workspace_size(c["rows"], c["vocab"], c["top"])
    elif c["kind"] == "select":
        size = B.select_kv_tokens_workspace_size(c["seqs"], c["heads"], s["max_len"])
    return B, desc, torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)


def _run_own(s):
    c = s["case"]
    if "handle" not in s:
        s["handle"] = _handle(s)
    B, desc, ws = s["handle"]
    if c["kind"] == "logprobs":
        x, o = s["logits"], s["out"]
        B.token_logprobs(x, B.SPD_F32 if c["dtype"] == "f32" else B.SPD_BF16, c["rows"], c["vocab"], x.stride(0), s["temperature"],
                         s["tokens"], c["top"], o["logprobs"], o["ranks"], o["entropy"], o["lse"], o.get("top_tokens"),
                         o.get("top_logprobs"), ws)
        return o
    if c["kind"] == "weights":
        B.accumulate_kv_weights(desc, s["q"], s["k"], s["new_starts"], s["kv_lens"], s["kv_starts"], s["pages"], s["lse"], s["total"],
                                s["max_new"], s["max_kv"], 1.0, s["weights"], s["out"], s["out"].stride(1), ws)
        return s["out"]
    if c["kind"] == "select":
        w, o = s["weights"], s["out"]
        B.select_kv_tokens(w, w.stride(1), c["seqs"], c["heads"], s["lens"], s["max_len"], s["budgets"], s["max_new"], c["sinks"],
                           c["recent"], o["source"], o["source"].stride(1), o["new_lens"], ws)
        return o
    B.compact_kv(desc, s["source"], s["source"].stride(0), s["source"].stride(1), s["new_lens"], s["max_new"], s["starts"], s["pages"],
                 s["k"], s["v"], s["out_starts"], s["out_pages"], s["k_out"], s["v_out"], s["weights"], s["weights_out"],
                 s["weights"].stride(1), s["lens"])
    return {"k": s["k_out"], "v": s["v_out"], "weights": s["weights_out"], "lens": s["lens"]}


# ---- the plain forms ----------------------------------------------------------------------------------------

def _which(starts, total):
    """For each of `total` packed places, the index of the range of `starts` that it lies in, and its place there."""
    t = torch.arange(total, device=DEV, dtype=torch.int32)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp_(max=starts.numel() - 2)
    return b, t - starts[b]


def _rank_keys(x):
    """Whole numbers of 64 bits that are in the order of x's last axis: larger values first, ties by the lower index."""
    bits = torch.where(x == 0, 0.0, x).view(torch.int32).long()  # (both zeros are one value)
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return bits * 2**31 + (2**31 - 1 - torch.arange(x.shape[-1], device=DEV))


def _plain_logprobs(s):
    c, x = s["case"], s["logits"].float()
    y = x / s["temperature"][:, None] if s["temperature"] is not None else x
    m = y.amax(1, keepdim=True)
    p = torch.exp(y - m)
    z = p.sum(1)
    lse = m[:, 0] + torch.log(z)
    at = s["tokens"].long()[:, None]
    got = {"logprobs": (y.gather(1, at) - m)[:, 0] - torch.log(z), "ranks": ((x > x.gather(1, at)).sum(1) + 1).to(torch.int32),
           "entropy": torch.log(z) + (p * (m - y)).sum(1) / z, "lse": lse}
    if c["top"]:
        top = torch.topk(_rank_keys(x), c["top"], dim=1, sorted=True)[1]
        got.update(top_tokens=top.to(torch.int32), top_logprobs=(y.gather(1, top) - m) - torch.log(z)[:, None])
    return got


def _padded(s, name, kv_starts, pages, most):
    """[sequences, most, heads, d] of a cache, in 32 bits (what lies past a sequence's end is another's)."""
    t = torch.arange(most, device=DEV)
    if pages is not None:
        page = pages[(kv_starts[:-1, None] + t // PAGE).clamp(max=pages.numel() - 1)]
        return s[name][page, :, t % PAGE].float()
    return s[name][(kv_starts[:-1, None] + t).clamp(max=s[name].shape[0] - 1)].float()


def _scores(s):
    """Scaled scores [sequences, kv heads, queries * group, tokens], and which of them count."""
    c, mq, mk = s["case"], s["max_new"], s["max_kv"]
    hq, hkv, d, n = c["hq"], c["hkv"], c["d"], c["seqs"]
    starts, kv_lens = s["new_starts"], s["kv_lens"]
    new = starts[1:] - starts[:-1]
    i, t = torch.arange(mq, device=DEV), torch.arange(mk, device=DEV)
    q = s["q"].float()[(starts[:-1, None] + i).clamp(max=s["total"] - 1)]                    # [n, mq, hq, d]
    q = q.unflatten(2, (hkv, -1)).permute(0, 2, 1, 3, 4).reshape(n, hkv, mq * (hq // hkv), d)
    k = _padded(s, "k", s["kv_starts"], s["pages"], mk)
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(d))
    seen = (i < new[:, None])[:, :, None] & (t < kv_lens[:, None])[:, None, :]
    if c["causal"]:
        seen = seen & (t <= (kv_lens - new)[:, None, None] + i[:, None])
    g = hq // hkv
    return x, seen[:, None, :, None, :].expand(n, 1, mq, g, mk).reshape(n, 1, mq * g, mk)


def _plain_weights(s):
    c, mq = s["case"], s["max_new"]
    n, hkv = c["seqs"], c["hkv"]
    x, seen = _scores(s)
    i = torch.arange(mq, device=DEV)
    lse = s["lse"][(s["new_starts"][:-1, None] + i).clamp(max=s["total"] - 1)]               # [n, mq, hq]
    lse = lse.unflatten(2, (hkv, -1)).permute(0, 2, 1, 3).reshape(n, hkv, -1)
    x.sub_(lse[..., None]).exp_().masked_fill_(~seen, 0.0)
    total = x.sum(2)
    if s["weights"] is not None:
        total = s["weights"] + total
    inside = torch.arange(s["max_kv"], device=DEV) < s["kv_lens"][:, None, None]
    return torch.where(inside, total, s["out"])


def _plain_source(weights, lens, budgets, sinks, recent, source):
    """`source` with the tokens that stay, each at its new place, and the new lengths."""
    n, heads, most = weights.shape
    room = source.shape[2]
    t = torch.arange(most, device=DEV)
    new = torch.minimum(lens, budgets)
    last = new.clamp(max=recent)
    first = torch.minimum(torch.full_like(new, sinks), new - last)
    ln, m, r, f = (v.long()[:, None, None] for v in (lens, new, last, first))
    keys = _rank_keys(weights)
    keys = torch.where((t < f) | (t >= ln - r), 2**62 - t, keys).masked_fill(t >= ln, -2**63)
    order = torch.topk(keys, room, dim=2, sorted=True)[1]
    stays = torch.zeros_like(keys, dtype=torch.bool).scatter_(2, order, (torch.arange(room, device=DEV) < m).expand_as(order))
    # the last ones keep their order at the end; what stays behind the others' new end fills the gaps before it
    early = t < ln - r
    moving = stays & early & (t >= m - r)
    behind = torch.full((n, heads, most + 1), most, dtype=torch.int64, device=DEV)
    behind.scatter_(2, torch.where(moving, moving.cumsum(2) - 1, most), t.expand_as(moving))
    j = torch.arange(room, device=DEV)
    here = stays[:, :, :room]
    gap = ~here & (j < m - r)
    fill = behind.gather(2, (gap.cumsum(2) - 1).clamp(min=0))
    got = torch.where(j >= m - r, j - m + ln, torch.where(gap, fill, j))
    return torch.where(j < m, got, source).to(torch.int32), new


def _plain_select(s):
    c = s["case"]
    source, new = _plain_source(s["weights"], s["lens"], s["budgets"], c["sinks"], c["recent"], s["out"]["source"])
    return {"source": source, "new_lens": new}


def _plain_compact(s):
    c, source = s["case"], s["source"].long()
    n, hkv, most = source.shape
    j = torch.arange(most, device=DEV)
    inside = j < s["new_lens"][:, None, None]
    inside, b, h, j = torch.broadcast_tensors(inside, torch.arange(n, device=DEV)[:, None, None], torch.arange(hkv, device=DEV)[:, None], j)
    b, h, j = b[inside], h[inside], j[inside]
    src = source[inside]
    for name in ("k", "v"):
        if s["pages"] is not None:
            page, to = s["pages"][s["starts"][b] + src // PAGE].long(), s["out_pages"][s["out_starts"][b] + j // PAGE].long()
            s[name + "_out"][to, h, j % PAGE] = s[name][page, h, src % PAGE]
        else:
            s[name + "_out"][s["out_starts"][b] + j, h] = s[name][s["starts"][b] + src, h]
    weights = torch.zeros_like(s["weights"])
    weights[b, h, j] = s["weights"][b, h, src]
    return {"k": s["k_out"], "v": s["v_out"], "weights": weights, "lens": s["new_lens"].clone()}


def run(state):
    if own:
        return _run_own(state)
    return {"logprobs": _plain_logprobs, "weights": _plain_weights, "select": _plain_select,
            "compact": _plain_compact}[state["case"]["kind"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(case):
    c, e = case, 4 if case.get("dtype") == "f32" else 2
    if c["kind"] == "logprobs":
        return {"bytes": c["rows"] * (c["vocab"] * e + 4 * (5 + c["hot"]) + 8 * c["top"]), "flops": 0}
    if c["kind"] == "weights":
        # sequences' new and cached lengths are paired at random: the sums of products go by the means
        new, past = (_spread(c[w + "_lo"], c[w + "_hi"], c["seqs"]) for w in ("new", "past"))
        pairs = sum(x * (sum(past) / len(past)) + (x * (x + 1) / 2 if c["causal"] else 0) for x in new)
        tokens = sum(past) + (sum(new) if c["causal"] else 0)
        byte = tokens * c["hkv"] * (c["d"] * e + 4 * (1 + c["sums"])) + sum(new) * c["hq"] * (c["d"] * e + 4)
        return {"bytes": byte, "flops": 2 * c["d"] * c["hq"] * pairs}
    lens = _spread(c["len_lo"], c["len_hi"], c["seqs"])
    new = [min(a, b) for a, b in zip(lens, _budgets(c, lens))]
    if c["kind"] == "select":
        return {"bytes": 4 * c["heads"] * (sum(lens) + sum(new)) + 12 * c["seqs"], "flops": 0}
    # in place only what comes from behind the new end moves; weights are read where their token moves and all written
    moved = sum(m * (n - m) / n for n, m in zip(lens, new) if n) if c["in_place"] else sum(new)
    weights = sum(new) + c["seqs"] * max(lens)
    return {"bytes": c["hkv"] * (moved * 4 * c["d"] * e + 4 * sum(new) + 4 * weights) + 8 * c["seqs"], "flops": 0}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _exact_logprobs(c, s):
    got = {k: None if v.dtype == torch.int32 else torch.empty(v.shape, dtype=torch.float64, device=DEV) for k, v in s["out"].items()}
    for r in range(c["rows"]):
        x = s["logits"][r].double()
        if c["hot"]:
            x = x / s["temperature"][r].double()
        logp = x - torch.logsumexp(x, 0)
        got["lse"][r] = torch.logsumexp(x, 0)
        got["logprobs"][r] = logp[s["tokens"][r].long()]
        got["entropy"][r] = -(torch.exp(logp) * logp).sum()
        if c["top"]:
            got["top_logprobs"][r] = torch.sort(logp, descending=True)[0][:c["top"]]
    return got


def _exact_weights(c, s):
    g, d = c["hq"] // c["hkv"], c["d"]
    out = s["out"].double()
    starts, kv_starts, lens = s["new_starts"].tolist(), s["kv_starts"].tolist(), s["kv_lens"].tolist()
    for b in range(c["seqs"]):
        n, length = starts[b + 1] - starts[b], lens[b]
        if length == 0:
            continue
        if c["page"]:
            keys = s["k"][s["pages"][kv_starts[b]:kv_starts[b + 1]].long()].transpose(1, 2).flatten(0, 1)[:length]
        else:
            keys = s["k"][kv_starts[b]:kv_starts[b] + length]
        for j in range(c["hkv"]):
            k = keys[:, j].double()
            total = s["weights"][b, j, :length].double() if s["weights"] is not None else torch.zeros(length, dtype=torch.float64, device=DEV)
            for first in range(0, n, 2048):
                q0, q1 = starts[b] + first, starts[b] + min(n, first + 2048)
                q = s["q"][q0:q1, j * g:j * g + g].double()
                p = torch.matmul(q.flatten(0, 1), k.t().contiguous()).div_(d ** 0.5)
                p.sub_(s["lse"][q0:q1, j * g:j * g + g].double().flatten()[:, None]).exp_()
                if c["causal"]:
                    limit = (length - n + torch.arange(first, first + q1 - q0, device=DEV)).repeat_interleave(g)
                    p[torch.arange(length, device=DEV)[None, :] > limit[:, None]] = 0.0
                total = total + p.sum(0)
            out[b, j, :length] = total
    return out


def _exact_compact(c, s):
    """A copy has one right value: that of the row that stays."""
    def rows(x):  # [pages, heads, 16, d] as [slots, heads, d]
        return x.transpose(1, 2).flatten(0, 1) if c["page"] else x

    def slots(starts, pages, b, at):
        return pages[starts[b] + at // PAGE].long() * PAGE + at % PAGE if c["page"] else starts[b] + at

    got = {"weights": torch.zeros(s["weights"].shape, dtype=torch.float64, device=DEV), "lens": None}
    olds = {name: rows(s[name]) for name in ("k", "v")}
    news = {name: rows(s[name + "_out"]).double() for name in ("k", "v")}
    for b, m in enumerate(s["new_lens"].tolist()):
        to = slots(s["out_starts"], s["out_pages"], b, torch.arange(m, device=DEV))
        for h in range(c["hkv"]):
            src = s["source"][b, h, :m].long()
            got["weights"][b, h, :m] = s["weights"][b, h, src].double()
            at = slots(s["starts"], s["pages"], b, src)
            for name in ("k", "v"):
                news[name][to, h] = olds[name][at, h].double()
    for name in ("k", "v"):
        got[name] = news[name].unflatten(0, (-1, PAGE)).transpose(1, 2).contiguous() if c["page"] else news[name]
    return got


def exact(case, seed):
    if case["kind"] == "select":
        return None  # whole numbers
    if case["kind"] == "logprobs" and case["rows"] * case["vocab"] > 2e8:
        return None
    s = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "weights": _exact_weights, "compact": _exact_compact}[case["kind"]](case, s)
