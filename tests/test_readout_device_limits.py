"""Sizes that the operators on a step's softmaxes do not take are refused where the plumbing is set up, not at the first step (no GPU needed)."""
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dev():
    from paper_2502_02534_amd import binding, device
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return device


def _attn(dev, n, hkv, room):
    """A decode call of n samples (one element's memory: nothing is read)."""
    from paper_2502_02534_amd import binding as B
    desc = B.make_desc(dtype=B.SPD_F32, num_q_heads=hkv, num_kv_heads=hkv, head_dim=64, num_prompts=1, num_samples=n)
    some = lambda *s, t=torch.float32: torch.zeros(1, dtype=t).expand(*s)  # noqa: E731
    i32 = lambda k: some(k, t=torch.int32)  # noqa: E731
    kv = some(n, room, hkv, 64)
    return dev.DeviceAttn(desc, some(n, hkv, 64), kv, kv, i32(1), i32(2), None, i32(2), kv, kv, i32(n), None, None, 4, room, some(n, hkv, 64),
                          some(n, hkv), i32(64))


@pytest.mark.parametrize("n,hkv,room", [
    (65537, 1, 1), (8193, 8, 2),         # more (sequence, KV head) pairs than compact_kv takes
    (60000, 1, 4500), (4096, 8, 8192),   # more tokens than accumulate_kv_weights has workgroups for
])
def test_eviction(dev, n, hkv, room):
    with pytest.raises(ValueError, match="more than"):
        dev.DeviceEviction(_attn(dev, n, hkv, room), 1)


def test_eviction_at_the_limits(dev):
    assert dev.DeviceEviction(_attn(dev, 65536, 1, 1), 1).weights.shape == (65536, 1, 1)
    assert dev.DeviceEviction(_attn(dev, 8192, 8, 64), 1).weights.shape == (8192, 8, 64)


@pytest.mark.parametrize("rows,vocab", [(1 << 22, 10), ((1 << 22) - 7, 10), (1 << 21, 20000)])
def test_logprobs(dev, rows, vocab, monkeypatch):
    monkeypatch.setattr(dev, "_on_one_gpu", lambda *t: True)
    with pytest.raises(ValueError, match="more than"):
        dev.DeviceLogprobs(torch.empty((rows, vocab), dtype=torch.bfloat16, device="meta"), torch.empty(rows, dtype=torch.int32, device="meta"))
