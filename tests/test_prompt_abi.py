"""What the prompt and logits operators refuse on the host, before any launch (no GPU needed: the pointers
are never dereferenced), and the launch plan of prompt_attn."""
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


def _attn(B, desc, q=P, k=P, v=P, qi=P, kl=P, ki=P, pages=P, total=0, mq=100, mk=100, out=P, lse=P, ws=P, size=1 << 40):
    return B.load().prompt_attn(None if desc is None else ctypes.byref(desc), q, k, v, qi, kl, ki, pages, total, mq, mk, out, lse,
                                ws, size, 0)


def test_prompt_attn_refuses(B):
    assert _attn(B, _desc(B)) == OK                                       # no queries: nothing to do, nothing launched
    assert _attn(B, None) == EINVAL
    for bad in (dict(num_kv_heads=0), dict(num_q_heads=0), dict(num_q_heads=30), dict(head_dim=0), dict(num_prompts=0),
                dict(q_stride=-8), dict(kv_stride=-8), dict(q_stride=32 * 128 + 4), dict(kv_stride=8 * 128 + 4),
                dict(q_stride=128), dict(kv_stride=128)):
        assert _attn(B, _desc(B, **bad)) == EINVAL, bad
        assert B.prompt_attn_workspace_size(_desc(B, **bad), 100, 100, 100) == 0, bad
    for bad in (dict(dtype=2), dict(head_dim=264), dict(head_dim=12), dict(page_size=32)):
        assert _attn(B, _desc(B, **bad)) == EUNSUPPORTED, bad
        assert B.prompt_attn_workspace_size(_desc(B, **bad), 100, 100, 100) == 0, bad
    for name in ("q", "k", "v", "qi", "kl", "ki", "out"):
        assert _attn(B, _desc(B), **{name: 0}) == EINVAL, name
    for name in ("q", "k", "v", "out"):
        assert _attn(B, _desc(B), **{name: P + 8}) == EINVAL, name
    for name in ("qi", "kl", "ki", "pages", "lse"):
        assert _attn(B, _desc(B), **{name: P + 2}) == EINVAL, name
    assert _attn(B, _desc(B, page_size=16), pages=0) == EINVAL
    assert _attn(B, _desc(B), pages=0, lse=0) == OK
    assert _attn(B, _desc(B), total=-1) == EINVAL and _attn(B, _desc(B), mq=-1) == EINVAL and _attn(B, _desc(B), mk=-1) == EINVAL
    assert _attn(B, _desc(B), total=1 << 31) == EUNSUPPORTED
    assert _attn(B, _desc(B), mk=1 << 31) == EUNSUPPORTED
    # few queries over many tokens are cut into splits, which need the workspace
    need = B.prompt_attn_workspace_size(_desc(B), 4, 1, 8192)
    assert need > 4 * 32 * 128 * 4
    for kw in (dict(ws=0), dict(ws=P + 64), dict(size=need // 2)):
        assert _attn(B, _desc(B), total=4, mq=1, mk=8192, **kw) == EWORKSPACE, kw
    # fp32 rows are 16 bytes from four elements on
    assert _attn(B, _desc(B, dtype=B.SPD_F32, q_stride=32 * 128 + 4, kv_stride=8 * 128 + 4)) == OK


def _tables(B, n=4, page=16, lens=P, hl=0, hi=0, hp=0, free=P, num_free=10, begin=0, mp=10, mt=10, pi=P, px=P, lo=P, ni=P, sm=P, fe=P,
            ws=P, size=1 << 20):
    return B.load().build_page_tables(n, page, lens, hl, hi, hp, free, num_free, begin, mp, mt, pi, px, lo, ni, sm, fe, ws, size, 0)


def test_build_page_tables_refuses(B):
    assert _tables(B, n=0) == EINVAL and _tables(B, n=-1) == EINVAL and _tables(B, page=0) == EINVAL
    assert _tables(B, num_free=-1) == EINVAL and _tables(B, mp=-1) == EINVAL and _tables(B, mt=-1) == EINVAL
    assert _tables(B, page=65537) == EUNSUPPORTED and _tables(B, mt=1 << 31) == EUNSUPPORTED and _tables(B, n=1 << 31) == EUNSUPPORTED
    for name in ("lens", "free", "pi", "px", "lo", "ni", "fe"):
        assert _tables(B, **{name: 0}) == EINVAL, name
        assert _tables(B, **{name: P + 1}) == EINVAL, name
    assert _tables(B, sm=P + 4) == EINVAL
    assert _tables(B, hl=P) == EINVAL and _tables(B, hl=P, hi=P) == EINVAL and _tables(B, hp=P) == EINVAL
    assert _tables(B, begin=P, fe=P) == EINVAL                             # one call's input and output
    assert _tables(B, ws=0) == EWORKSPACE and _tables(B, ws=P + 4) == EWORKSPACE and _tables(B, size=8) == EWORKSPACE
    assert B.build_page_tables_workspace_size(0) == 0 and B.build_page_tables_workspace_size(-3) == 0
    assert B.build_page_tables_workspace_size(1) >= 4 and B.build_page_tables_workspace_size(10000) >= 40000


def _write(B, desc, k=P, v=P, slots=P, tokens=0, pages=10, kp=P, vp=P):
    return B.load().write_prompt_kv(None if desc is None else ctypes.byref(desc), k, v, slots, tokens, pages, kp, vp, 0)


def test_write_prompt_kv_refuses(B):
    assert _write(B, _desc(B, page_size=16)) == OK and _write(B, _desc(B), tokens=5, pages=0) == OK
    assert _write(B, None) == EINVAL
    for name in ("k", "v", "slots", "kp", "vp"):
        assert _write(B, _desc(B), **{name: 0}) == EINVAL, name
        assert _write(B, _desc(B), **{name: P + 4}) == EINVAL, name
    assert _write(B, _desc(B), tokens=-1) == EINVAL and _write(B, _desc(B), pages=-1) == EINVAL
    assert _write(B, _desc(B, kv_stride=100)) == EINVAL and _write(B, _desc(B, kv_stride=512)) == EINVAL
    assert _write(B, _desc(B, page_size=8)) == EUNSUPPORTED and _write(B, _desc(B, head_dim=512)) == EUNSUPPORTED
    assert _write(B, _desc(B), tokens=1 << 31) == EUNSUPPORTED


def test_mark_prompt_tokens_refuses(B):
    f = lambda tokens=P, indptr=P, n=2, vocab=100, bits=P, stride=4, acc=0: B.load().mark_prompt_tokens(  # noqa: E731
        tokens, indptr, n, vocab, bits, stride, acc, 0)
    for kw in (dict(tokens=0), dict(indptr=0), dict(bits=0), dict(n=0), dict(vocab=0), dict(stride=3), dict(tokens=P + 1),
               dict(bits=P + 2)):
        assert f(**kw) == EINVAL, kw
    assert f(vocab=(1 << 20) + 1, stride=1 << 20) == EUNSUPPORTED and f(n=1 << 31) == EUNSUPPORTED


def test_penalize_logits_refuses(B):
    def f(logits=P, dtype=0, rows=0, vocab=100, stride=100, out=2 * P, out_stride=100, pen=True, **parts):
        rec = B.Penalties(**parts) if pen else None
        return B.load().penalize_logits(logits, dtype, rows, vocab, stride, None if rec is None else ctypes.byref(rec), out, out_stride, 0)

    assert f() == OK                                                       # no rows
    for kw in (dict(logits=0), dict(out=0), dict(pen=False), dict(rows=-1), dict(vocab=0), dict(stride=99), dict(out_stride=99),
               dict(logits=P + 2), dict(out=P + 2), dict(logits=P, out=P, out_stride=101), dict(logits=P, out=P, dtype=1),
               dict(tokens=P), dict(tokens=P, token_lens=P, max_tokens=-1), dict(bias_tokens=P), dict(bias_tokens=P, bias_indptr=P),
               dict(prompt_bits=P, prompt_bits_stride=3), dict(allowed_bits=P, allowed_stride=3), dict(repetition=P + 1),
               dict(allowed_of_row=P + 2)):
        assert f(**kw) == EINVAL, kw
    assert f(dtype=2) == EUNSUPPORTED
    assert f(vocab=(1 << 30) + 1, stride=1 << 31, out_stride=1 << 31) == EUNSUPPORTED
    assert f(tokens=P, token_lens=P, max_tokens=(1 << 24) + 1) == EUNSUPPORTED
    assert f(dtype=1, logits=P + 2) == OK and f(logits=P, out=P) == OK


def test_binding_raises_with_the_entry_point_s_name(B):
    desc = _desc(B, head_dim=12)
    with pytest.raises(B.SpdError, match="prompt_attn") as e:
        B.prompt_attn(desc, None, None, None, None, None, None, None, 1, 1, 1, None, None, None, 0)
    assert e.value.status == EUNSUPPORTED
    with pytest.raises(B.SpdError, match="write_prompt_kv"):
        B.write_prompt_kv(desc, None, None, None, 1, 1, None, None, 0)
    with pytest.raises(B.SpdError, match="build_page_tables"):
        B.build_page_tables(0, 16, None, None, None, None, None, 0, None, 0, 0, None, None, None, None, None, None, None, 0)
    with pytest.raises(B.SpdError, match="mark_prompt_tokens"):
        B.mark_prompt_tokens(None, None, 1, 10, None, 1, stream=0)
    with pytest.raises(B.SpdError, match="penalize_logits"):
        B.penalize_logits(None, 0, 1, 10, 10, B.make_penalties(), None, 10, 0)
