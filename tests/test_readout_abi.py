"""What the operators on a step's softmaxes refuse on the host, before any launch (no GPU needed: the pointers are never dereferenced)."""
import ctypes
import os

import pytest

P = 4096          # a pointer, never dereferenced
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def B():
    from paper_2502_02534_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    binding.load()
    return binding


def _desc(B, **kw):
    a = dict(dtype=B.SPD_BF16, num_q_heads=32, num_kv_heads=8, head_dim=128, num_prompts=4)
    a.update(kw)
    return B.make_prompt_desc(**a)


def _logprobs(B, x=P, dtype=1, rows=0, vocab=1000, stride=1000, t=P, tokens=P, top=5, lp=P, rk=P, en=P, ls=P, tt=P, tl=P, ws=P, size=1 << 40):
    return B.load().token_logprobs(x, dtype, rows, vocab, stride, t, tokens, top, lp, rk, en, ls, tt, tl, ws, size, 0)


def test_token_logprobs_refuses(B):
    assert _logprobs(B) == OK                                             # no rows: nothing to do
    assert _logprobs(B, x=0) == EINVAL and _logprobs(B, rows=-1) == EINVAL and _logprobs(B, vocab=0) == EINVAL
    assert _logprobs(B, stride=999) == EINVAL and _logprobs(B, top=-1) == EINVAL
    assert _logprobs(B, top=6, vocab=5, stride=5) == EINVAL and _logprobs(B, top=65) == EUNSUPPORTED
    assert _logprobs(B, dtype=2) == EUNSUPPORTED and _logprobs(B, vocab=(1 << 30) + 1, stride=1 << 31) == EUNSUPPORTED
    assert _logprobs(B, rows=1 << 22) == EUNSUPPORTED
    assert _logprobs(B, tokens=0) == EINVAL and _logprobs(B, tokens=0, lp=0) == EINVAL and _logprobs(B, tokens=0, rk=0) == EINVAL
    assert _logprobs(B, tokens=0, lp=0, rk=0) == OK and _logprobs(B, t=0, en=0, ls=0, tt=0, tl=0) == OK
    assert _logprobs(B, x=P + 1) == EINVAL and _logprobs(B, x=P + 2, dtype=0) == EINVAL and _logprobs(B, x=P + 2) == OK
    for name in ("t", "tokens", "lp", "rk", "en", "ls", "tt", "tl"):
        assert _logprobs(B, **{name: P + 2}) == EINVAL, name
    size = B.token_logprobs_workspace_size
    assert size(64, 128256, 20) > 0 and size(-1, 10, 1) == 0 and size(1, 0, 0) == 0 and size(1, 10, 11) == 0 and size(1, 100, 65) == 0


def _weights(B, desc, q=P, k=P, qi=P, kl=P, ki=P, pages=P, lse=P, total=0, mq=0, mk=0, decay=1.0, w=P, out=P, stride=1000, ws=P, size=1 << 40):
    return B.load().accumulate_kv_weights(None if desc is None else ctypes.byref(desc), q, k, qi, kl, ki, pages, lse, total, mq, mk, decay, w,
                                          out, stride, ws, size, 0)


def test_accumulate_kv_weights_refuses(B):
    assert _weights(B, _desc(B)) == OK                                    # no tokens: nothing to do
    assert _weights(B, None) == EINVAL
    for bad in (dict(num_kv_heads=0), dict(num_q_heads=30), dict(head_dim=0), dict(num_prompts=0), dict(q_stride=-8), dict(kv_stride=128)):
        assert _weights(B, _desc(B, **bad)) == EINVAL, bad
        assert B.accumulate_kv_weights_workspace_size(_desc(B, **bad), 10, 10, 10) == 0, bad
    for bad in (dict(dtype=2), dict(head_dim=264), dict(head_dim=12), dict(page_size=32)):
        assert _weights(B, _desc(B, **bad)) == EUNSUPPORTED, bad
    for name in ("q", "k", "qi", "kl", "ki", "lse", "out"):
        assert _weights(B, _desc(B), **{name: 0}) == EINVAL, name
    for name in ("q", "k"):
        assert _weights(B, _desc(B), **{name: P + 8}) == EINVAL, name
    for name in ("qi", "kl", "ki", "pages", "lse", "w", "out"):
        assert _weights(B, _desc(B), **{name: P + 2}) == EINVAL, name
    assert _weights(B, _desc(B, page_size=16), pages=0) == EINVAL and _weights(B, _desc(B), pages=0, w=0) == OK
    assert _weights(B, _desc(B), total=-1) == EINVAL and _weights(B, _desc(B), mq=-1) == EINVAL and _weights(B, _desc(B), mk=-1) == EINVAL
    assert _weights(B, _desc(B), mk=1001) == EINVAL
    assert _weights(B, _desc(B), mk=(1 << 30) + 1, stride=1 << 31) == EUNSUPPORTED and _weights(B, _desc(B), total=1 << 27) == EUNSUPPORTED
    assert _weights(B, _desc(B, num_prompts=1 << 20), mk=1000) == EUNSUPPORTED
    assert B.accumulate_kv_weights_workspace_size(_desc(B), 64, 64, 8192) > 0


def _select(B, w=P, stride=1000, seqs=4, heads=2, lens=P, mk=1000, budgets=P, mn=500, sinks=0, recent=0, src=P, ss=1000, new=P, ws=P, size=1 << 40):
    return B.load().select_kv_tokens(w, stride, seqs, heads, lens, mk, budgets, mn, sinks, recent, src, ss, new, ws, size, 0)


def test_select_kv_tokens_refuses(B):
    for name in ("w", "lens", "src", "new"):
        assert _select(B, **{name: 0}) == EINVAL, name
    for name in ("w", "lens", "budgets", "src", "new"):
        assert _select(B, **{name: P + 2}) == EINVAL, name
    for bad in (dict(seqs=0), dict(heads=0), dict(mk=-1), dict(mn=-1), dict(sinks=-1), dict(recent=-1), dict(stride=999), dict(ss=499)):
        assert _select(B, **bad) == EINVAL, bad
    assert _select(B, mk=(1 << 24) + 1, stride=1 << 25) == EUNSUPPORTED and _select(B, seqs=1 << 22) == EUNSUPPORTED
    size = B.select_kv_tokens_workspace_size
    assert size(4, 2, 1000) > 0 and size(0, 2, 10) == 0 and size(4, 0, 10) == 0 and size(1, 1, -1) == 0 and size(1, 1, 1 << 25) == 0


def _compact(B, desc, src=P, ss=1000, hs=500, new=P, mn=500, ki=P, kp=P, k=P, v=2 * P, oi=2 * P, op=2 * P, ko=3 * P, vo=4 * P, w=P, wo=P, stride=1000,
             lens=P):
    return B.load().compact_kv(None if desc is None else ctypes.byref(desc), src, ss, hs, new, mn, ki, kp, k, v, oi, op, ko, vo, w, wo, stride,
                               lens, 0)


def test_compact_kv_refuses(B):
    d = _desc(B, page_size=16)
    assert _compact(B, None) == EINVAL
    for bad in (dict(num_kv_heads=0), dict(head_dim=0), dict(num_prompts=0), dict(kv_stride=128)):
        assert _compact(B, _desc(B, **bad)) == EINVAL, bad
    for bad in (dict(dtype=2), dict(head_dim=264), dict(head_dim=12), dict(page_size=32)):
        assert _compact(B, _desc(B, **bad)) == EUNSUPPORTED, bad
    for name in ("src", "new", "ki", "oi", "k", "v", "ko", "vo", "kp", "op"):
        assert _compact(B, d, **{name: 0}) == EINVAL, name
    for name in ("k", "v", "ko", "vo"):
        assert _compact(B, d, **{name: 5 * P + 8}) == EINVAL, name
    for name in ("src", "new", "ki", "kp", "oi", "op", "lens"):
        assert _compact(B, d, **{name: P + 2}) == EINVAL, name
    assert _compact(B, d, w=P + 2, wo=P + 2) == EINVAL and _compact(B, d, w=0) == EINVAL and _compact(B, d, wo=0) == EINVAL
    for bad in (dict(mn=-1), dict(ss=-1), dict(hs=-1), dict(ss=499), dict(hs=499), dict(stride=499)):
        assert _compact(B, d, **bad) == EINVAL, bad
    assert _compact(B, d, vo=3 * P) == EINVAL                               # keys and values into one place
    assert _compact(B, d, oi=P, op=P, ko=P) == EINVAL                       # half in place
    assert _compact(B, _desc(B, num_prompts=1 << 20)) == EUNSUPPORTED
    assert _compact(B, d, mn=(1 << 30) + 1, ss=1 << 31, hs=1 << 31, stride=1 << 31) == EUNSUPPORTED
