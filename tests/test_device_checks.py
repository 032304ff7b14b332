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
