"""What the device plumbing refuses before a launch (no GPU needed: a refusal comes before anything is read)."""
import dataclasses
import os

import pytest

torch = pytest.importorskip("torch")

HQ, HKV, D, TOKENS = 8, 2, 64, 40


@pytest.fixture(scope="module")
def dev():
    from paper_2502_02534_amd import binding, device
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return device


def _tables(dev, **kw):
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    t = dev.PageTables(i32(4), i32(6), i32(3), i32(4), torch.zeros(TOKENS, dtype=torch.int64), i32(1))
    return dataclasses.replace(t, **kw)


def _prompts(dev, dtype=torch.bfloat16, tables=None, **kw):
    draw = lambda *shape: torch.zeros(shape, dtype=dtype)  # noqa: E731
    a = dict(q=draw(TOKENS, HQ, D), k=draw(TOKENS, HKV, D), v=draw(TOKENS, HKV, D), k_pool=draw(6, HKV, 16, D),
             v_pool=draw(6, HKV, 16, D))
    a.update(kw)
    return dev.DevicePrompts(tables or _tables(dev), a["q"], a["k"], a["v"], a["k_pool"], a["v_pool"], 20, 20)


def test_prompts_that_are_sound_get_as_far_as_the_device(dev):
    with pytest.raises(ValueError, match="one GPU"):
        _prompts(dev)
    wide = torch.zeros((TOKENS, (HQ + 2 * HKV) * D))
    parts = dict(q=wide[:, :HQ * D].unflatten(1, (HQ, D)), k=wide[:, HQ * D:(HQ + HKV) * D].unflatten(1, (HKV, D)),
                 v=wide[:, (HQ + HKV) * D:].unflatten(1, (HKV, D)))
    with pytest.raises(ValueError, match="one GPU"):
        _prompts(dev, torch.float32, **parts)
    with pytest.raises(ValueError, match="one GPU"):  # one token's stride means nothing
        _prompts(dev, torch.float32, q=parts["q"][:1], k=torch.zeros(1, HKV, D), v=parts["v"][:1])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_prompts_of_other_types(dev, dtype):
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        _prompts(dev, dtype)


@pytest.mark.parametrize("name", ["k", "v", "k_pool", "v_pool"])
def test_prompts_of_mixed_types(dev, name):
    shape = (6, HKV, 16, D) if "pool" in name else (TOKENS, HKV, D)
    with pytest.raises(ValueError, match="q's type"):
        _prompts(dev, **{name: torch.zeros(shape)})


def test_keys_and_values_of_different_strides(dev):
    wide = torch.zeros((TOKENS, 3 * HKV * D), dtype=torch.bfloat16)
    part = wide[:, :HKV * D].unflatten(1, (HKV, D))
    for kw in (dict(k=part), dict(v=part)):
        with pytest.raises(ValueError, match="one token stride"):
            _prompts(dev, **kw)


def test_heads_or_channels_that_do_not_follow_one_another(dev):
    b16 = dict(dtype=torch.bfloat16)
    turned = torch.zeros((HKV, TOKENS, D), **b16).transpose(0, 1)
    apart = torch.zeros((TOKENS, HKV, 2 * D), **b16)[:, :, :D]
    every_other = torch.zeros((TOKENS, HKV, 2 * D), **b16)[:, :, ::2]
    for x in (turned, apart, every_other):
        for kw in (dict(k=x), dict(v=x), dict(k=x, v=x)):
            with pytest.raises(ValueError, match="follow one another"):
                _prompts(dev, **kw)
    with pytest.raises(ValueError, match="q's heads"):
        _prompts(dev, q=torch.zeros((HQ, TOKENS, D), **b16).transpose(0, 1))


def test_tokens_that_share_a_row(dev):
    for name, heads in (("q", HQ), ("k", HKV), ("v", HKV)):
        with pytest.raises(ValueError, match="overlap"):
            _prompts(dev, **{name: torch.zeros((1, heads, D), dtype=torch.bfloat16).expand(TOKENS, -1, -1)})


@pytest.mark.parametrize("name,shape", [("k", (TOKENS - 1, HKV, D)), ("v", (TOKENS, HKV + 1, D)), ("v", (TOKENS - 1, HKV, D)),
                                        ("q", (TOKENS + 1, HQ, D)), ("q", (TOKENS, HQ, D + 8)), ("q", (TOKENS, HQ * D))])
def test_shapes_that_do_not_go_together(dev, name, shape):
    with pytest.raises(ValueError, match="kv_heads"):
        _prompts(dev, **{name: torch.zeros(shape, dtype=torch.bfloat16)})


@pytest.mark.parametrize("name", ["k_pool", "v_pool"])
@pytest.mark.parametrize("shape", [(6, HKV, 32, D), (6, 16, HKV, D), (6, HKV, 16, D + 8), (96, HKV, D)])
def test_pools_of_another_layout(dev, name, shape):
    with pytest.raises(ValueError, match="pools are"):
        _prompts(dev, **{name: torch.zeros(shape, dtype=torch.bfloat16)})


def test_pools_of_different_sizes_or_strides(dev):
    with pytest.raises(ValueError, match="pools are"):
        _prompts(dev, v_pool=torch.zeros((5, HKV, 16, D), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="pools are"):
        _prompts(dev, v_pool=torch.zeros((6, 2 * HKV, 16, D), dtype=torch.bfloat16)[:, ::2])


def test_tables_that_do_not_fit(dev):
    for slots in (None, torch.zeros(TOKENS - 1, dtype=torch.int64)):
        with pytest.raises(ValueError, match="slot for every token"):
            _prompts(dev, tables=_tables(dev, slots=slots))
    with pytest.raises(ValueError, match="16 tokens"):
        _prompts(dev, tables=_tables(dev, page_size=64))
    for kw in (dict(slots=torch.zeros(TOKENS, dtype=torch.int32)), dict(lens=torch.zeros(3, dtype=torch.int64)),
               dict(new_indptr=torch.zeros(3, dtype=torch.int32)), dict(page_indptr=torch.zeros(8, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError, match="int32"):
            _prompts(dev, tables=_tables(dev, **kw))


ROWS, VOCAB = 3, 100
WORDS = 4


def _shape(dev, raw=None, to=None, **penalties):
    logits = torch.zeros((ROWS, VOCAB)) if to is None else to
    sampler = dev.DeviceSampler(logits, *(torch.zeros(ROWS) for _ in range(3)), torch.full((ROWS,), 5, dtype=torch.int32), torch.zeros(256))
    q = torch.zeros((2, ROWS, 4, 8))
    try:
        # (refused before the rest of the loop is looked at)
        dev.DecodeLoop(None, sampler, q, q, q, torch.zeros((2, ROWS)), raw_logits=torch.zeros((ROWS, VOCAB)) if raw is None else raw,
                       penalties=penalties)
    finally:
        assert bool((sampler.tokens == 5).all())


def test_penalties_that_are_sound_get_as_far_as_the_device(dev):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="one GPU"):
        _shape(dev)
    with pytest.raises(ValueError, match="one GPU"):
        _shape(dev, torch.zeros((ROWS, VOCAB + 7), dtype=torch.bfloat16)[:, :VOCAB], torch.zeros((ROWS, VOCAB + 3))[:, :VOCAB],
               repetition=torch.ones(ROWS), frequency=None, prompt_bits=i32(2, WORDS + 1), prompt_of_row=i32(ROWS), allowed_bits=i32(ROWS, WORDS),
               bias_indptr=i32(ROWS + 1), bias_tokens=i32(5), bias_values=torch.zeros(5))


def test_raw_logits_that_are_not_the_sampler_s(dev):
    for dtype in (torch.float16, torch.float64):
        with pytest.raises(ValueError, match="bfloat16 or float32"):
            _shape(dev, torch.zeros((ROWS, VOCAB), dtype=dtype))
    for shape in ((ROWS + 1, VOCAB), (ROWS - 1, VOCAB), (ROWS, VOCAB + 1), (VOCAB,)):
        with pytest.raises(ValueError, match="shape of the sampler"):
            _shape(dev, torch.zeros(shape))
    with pytest.raises(ValueError, match="shape of the sampler"):
        _shape(dev, to=torch.zeros((ROWS, VOCAB), dtype=torch.bfloat16))
    for bad in (torch.zeros((VOCAB, ROWS)).t(), torch.zeros((ROWS, 2 * VOCAB))[:, ::2], torch.zeros((1, VOCAB)).expand(ROWS, -1)):
        with pytest.raises(ValueError, match="contiguous"):
            _shape(dev, bad)
        with pytest.raises(ValueError, match="contiguous"):
            _shape(dev, to=bad)


@pytest.mark.parametrize("name", ["repetition", "frequency", "presence", "prompt_of_row", "allowed_of_row", "bias_indptr"])
def test_penalties_without_an_entry_for_every_row(dev, name):
    dtype = torch.int32 if "row" in name or "indptr" in name else torch.float32
    more = {"bias_tokens": torch.zeros(0, dtype=torch.int32), "bias_values": torch.zeros(0)} if "bias" in name else {}
    n = ROWS + ("indptr" in name)
    for bad in (torch.zeros(n - 1, dtype=dtype), torch.zeros(n, dtype=torch.int64), torch.zeros(2 * n, dtype=dtype)[::2],
                torch.zeros(1, dtype=dtype).expand(n)):
        with pytest.raises(ValueError, match=name):
            _shape(dev, **{name: bad}, **more)


@pytest.mark.parametrize("name", ["prompt_bits", "allowed_bits"])
def test_bits_that_do_not_fit(dev, name):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    for bad in (i32(ROWS, WORDS - 1), i32(ROWS - 1, WORDS), i32(ROWS * WORDS), i32(WORDS, ROWS).t(), i32(ROWS, WORDS).long(),
                i32(1, WORDS).expand(ROWS, -1)):
        with pytest.raises(ValueError, match=name):
            _shape(dev, **{name: bad})


def test_penalties_that_a_loop_does_not_take(dev):
    for name in ("tokens", "token_lens", "temperature"):
        with pytest.raises(ValueError, match=name):
            _shape(dev, **{name: torch.zeros(ROWS, dtype=torch.int32)})
    for kw in (dict(bias_tokens=torch.zeros(2, dtype=torch.int32)), dict(bias_values=torch.zeros(2)),
               dict(bias_indptr=torch.zeros(4, dtype=torch.int32), bias_tokens=torch.zeros(2, dtype=torch.int32), bias_values=torch.zeros(1))):
        with pytest.raises(ValueError, match="go together"):
            _shape(dev, **kw)


def test_lists_of_requests_of_other_types(dev):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    lens, free = i32(5, 40, 3), i32(*range(10))
    held = dev.PageTables(i32(0, 1, 2, 3), i32(7, 8, 9), i32(4, 4, 1), i32(0, 0, 0, 0), None, i32(0))
    with pytest.raises(ValueError, match="one GPU"):
        dev.build_tables(lens, free, 8, 60)
    with pytest.raises(ValueError, match="one GPU"):
        dev.build_tables(lens, free, 8, 60, held=held, free_begin=i32(0))
    for bad in (lens.long(), lens.float(), i32(5, 0, 40, 0, 3, 0)[::2], i32()):
        with pytest.raises(ValueError, match="lens"):
            dev.build_tables(bad, free, 8, 60)
    with pytest.raises(ValueError, match="free_pages"):
        dev.build_tables(lens, free.long(), 8, 60)
    for bad in (i32(0).long(), i32()):
        with pytest.raises(ValueError, match="free_begin"):
            dev.build_tables(lens, free, 8, 60, free_begin=bad)
    for kw in (dict(lens=i32(4, 4)), dict(page_size=64)):
        with pytest.raises(ValueError, match="same requests"):
            dev.build_tables(lens, free, 8, 60, held=dataclasses.replace(held, **kw))
    for kw in (dict(lens=held.lens.long()), dict(page_indptr=i32(0, 1, 2)), dict(page_indices=held.page_indices.long())):
        with pytest.raises(ValueError, match="held"):
            dev.build_tables(lens, free, 8, 60, held=dataclasses.replace(held, **kw))


def test_packed_counts_of_other_types_or_alone(dev):
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="one GPU"):
        _prompts(dev, tables=_tables(dev, packed_indptr=i32(4), packed_lens=i32(3)))
    for kw in (dict(packed_indptr=i32(4)), dict(packed_lens=i32(3))):
        with pytest.raises(ValueError, match="go together"):
            _prompts(dev, tables=_tables(dev, **kw))
    for kw in (dict(packed_indptr=i32(3), packed_lens=i32(3)), dict(packed_indptr=i32(4).long(), packed_lens=i32(3))):
        with pytest.raises(ValueError, match="int32"):
            _prompts(dev, tables=_tables(dev, **kw))


def test_raw_logits_that_are_shaped_where_they_lie(dev):
    """The second step would shape what the first one left."""
    x = torch.zeros((ROWS, VOCAB))
    wide = torch.zeros((ROWS, 2 * VOCAB))
    both = torch.zeros((2 * ROWS, VOCAB))
    for raw, to in ((x, x), (wide[:, :VOCAB], wide[:, 50:150]), (both[:ROWS], both[ROWS - 1:-1]), (x.view(torch.bfloat16)[:, :VOCAB], x)):
        with pytest.raises(ValueError, match="share memory"):
            _shape(dev, raw, to)
    with pytest.raises(ValueError, match="one GPU"):
        _shape(dev, both[:ROWS], both[ROWS:])


def test_a_sampler_without_a_token_for_every_row(dev):
    """The record of its tokens is the rows' history."""
    for tokens in (torch.full((ROWS - 1,), 5, dtype=torch.int32), torch.full((ROWS,), 5), torch.full((2 * ROWS,), 5, dtype=torch.int32)[::2]):
        sampler = dev.DeviceSampler(torch.zeros((ROWS, VOCAB)), *(torch.zeros(ROWS) for _ in range(3)), tokens, torch.zeros(256))
        q = torch.zeros((2, ROWS, 4, 8))
        with pytest.raises(ValueError, match="token for every row"):
            dev.DecodeLoop(None, sampler, q, q, q, torch.zeros((2, ROWS)), raw_logits=torch.zeros((ROWS, VOCAB)), penalties={})
