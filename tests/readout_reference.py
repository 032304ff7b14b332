"""Plain forms, in 64 bits and one element after another, of the operators on what a step's softmaxes say."""
import math

import torch

PAGE = 16


def logprobs(x, temperature, token, top):
    """One row of float64 logits: log probability and rank of `token`, entropy, lse, the `top` tokens and their log probabilities."""
    t = 1.0 if temperature == 0 else temperature
    y = x / t
    m = y.max()
    if m == -math.inf:
        logp, lse, entropy = torch.full_like(y, -math.inf), -math.inf, 0.0
    else:
        d = (x - x.max()) / t  # (no overflow where the logits are the type's lowest value)
        log_z = math.log(float(torch.exp(d).sum()))
        logp, lse = d - log_z, float(m) + log_z
        p = torch.exp(logp)
        entropy = -float((p * logp)[p > 0].sum())
    known = 0 <= token < x.numel()
    order = sorted(range(x.numel()), key=lambda i: (-float(x[i]), i))[:top]
    return {"logprob": float(logp[token]) if known else -math.inf, "rank": int((x > x[token]).sum()) + 1 if known else 0,
            "entropy": entropy, "lse": lse, "top_tokens": order, "top_logprobs": [float(logp[i]) for i in order]}


def kept(weights, n, budget, sinks, recent):
    """Places of one row after selection: entry i is the token that place i gets."""
    m = max(0, min(n, budget))
    if m == n:
        return list(range(n))
    r = min(recent, m)
    f = min(sinks, m - r)
    weight = lambda t: -math.inf if math.isnan(weights[t]) else weights[t]  # noqa: E731
    # (a NaN below -inf)
    middle = sorted(range(f, n - r), key=lambda t: (math.isnan(weights[t]), -weight(t), t))[:m - f - r]
    stay = set(range(f)) | set(middle)
    early = m - r
    fill = [t for t in sorted(stay) if t >= early]
    places = [t if t in stay else fill.pop(0) for t in range(early)]
    assert not fill
    return places + list(range(n - r, n))


def slots(indptr, pages, b, t):
    """Row of token t of sequence b: (page, place in it), or a row number."""
    if pages is None:
        return int(indptr[b]) + t
    return int(pages[int(indptr[b]) + t // PAGE]), t % PAGE


def row(pool, at, head):
    return pool[at[0], head, at[1]] if isinstance(at, tuple) else pool[at, head]


def weights(q, k_row, query_indptr, kv_lens, lse, causal, scale, decay, old, out, hkv):
    """Accumulated weights of every token, and the largest scale * sum |q k| that went into each sequence's.  k_row(b, t, j):
    the key; old: [B, Hkv, stride] or None; out: what places without a token hold."""
    out = out.double().clone()
    sizes = torch.zeros(len(kv_lens), dtype=torch.float64)
    g = q.shape[1] // hkv
    for b, length in enumerate(int(x) for x in kv_lens):
        if length == 0:
            continue
        q0, n = int(query_indptr[b]), int(query_indptr[b + 1]) - int(query_indptr[b])
        for j in range(hkv):
            k = torch.stack([k_row(b, t, j) for t in range(length)]).double()
            total = torch.zeros(length, dtype=torch.float64)
            for i in range(n):
                see = max(0, min(length, length - n + i + 1)) if causal else length
                for h in range(j * g, j * g + g):
                    x = float(lse[q0 + i, h])
                    if x == -math.inf or see == 0:
                        continue
                    qi = q[q0 + i, h].double()
                    sizes[b] = max(sizes[b], float((k[:see].abs() @ qi.abs()).max()) * scale)
                    total[:see] += torch.exp(k[:see] @ qi * scale - x)
            out[b, j, :length] = total + (decay * old[b, j, :length].double() if old is not None and decay != 0 else 0.0)
    return out, sizes
