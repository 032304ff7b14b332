"""What the device plumbing of log probabilities and eviction refuses before a launch (no GPU needed)."""
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


def _logprobs(dev, **kw):
    a = dict(logits=torch.zeros(4, 100), tokens=torch.zeros(4, dtype=torch.int32), temperature=torch.ones(4), num_top=5)
    a.update(kw)
    return dev.DeviceLogprobs(**a)


@pytest.mark.parametrize("kw,said", [
    (dict(logits=torch.zeros(4, 100, dtype=torch.float16)), "bfloat16 or float32"), (dict(logits=torch.zeros(400)), "rows, vocab"),
    (dict(logits=torch.zeros(100, 4).t()), "contiguous"), (dict(logits=torch.zeros(1, 100).expand(4, 100)), "contiguous"),
    (dict(tokens=torch.zeros(4, dtype=torch.int64)), "int32"), (dict(tokens=torch.zeros(3, dtype=torch.int32)), "every row"),
    (dict(tokens=torch.zeros(8, dtype=torch.int32)[::2]), "int32"), (dict(temperature=torch.ones(4, dtype=torch.float64)), "float32"),
    (dict(temperature=torch.ones(3)), "every row"), (dict(num_top=-1), "num_top"), (dict(num_top=65), "num_top"),
    (dict(logits=torch.zeros(4, 3)), "num_top"), (dict(), "one GPU")])
def test_logprobs(dev, kw, said):
    with pytest.raises(ValueError, match=said):
        _logprobs(dev, **kw)


def _attn(dev, n=6, hq=8, hkv=2, d=64, room=48, page=0):
    from paper_2502_02534_amd import binding as B
    desc = B.make_desc(dtype=B.SPD_F32, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, num_prompts=1, num_samples=n, page_size=page)
    i32 = lambda k: torch.zeros(k, dtype=torch.int32)  # noqa: E731
    kv = torch.zeros(n, room, hkv, d)
    return dev.DeviceAttn(desc, torch.zeros(n, hq, d), kv, kv, i32(1), i32(2), None, i32(2), kv, kv, i32(n), None, None, 4, room,
                          torch.zeros(n, hq, d), torch.zeros(n, hq), i32(64))


def test_eviction(dev):
    for kw in (dict(budget=0), dict(budget=49), dict(budget=-3)):
        with pytest.raises(ValueError, match="budget"):
            dev.DeviceEviction(_attn(dev), **kw)
    for kw in (dict(sinks=-1), dict(recent=-1)):
        with pytest.raises(ValueError, match="counts"):
            dev.DeviceEviction(_attn(dev), 16, **kw)
    e = dev.DeviceEviction(_attn(dev), 16)
    assert e.starts.tolist() == [48 * i for i in range(7)] and float(e.weights.abs().sum()) == 0.0


def test_loop_takes_its_own(dev):
    """Log probabilities of other tokens than the sampler's, and an eviction of another call."""
    attn, other = _attn(dev), _attn(dev)
    sampler = dev.DeviceSampler(torch.zeros(6, 50), torch.ones(6), torch.ones(6), torch.zeros(6), torch.zeros(6, dtype=torch.int32), torch.zeros(1))
    steps = lambda *s: torch.zeros(s)  # noqa: E731
    args = (attn, sampler, steps(3, 6, 8, 64), steps(3, 6, 2, 64), steps(3, 6, 2, 64), steps(3, 6))
    with pytest.raises(ValueError, match="attention call"):
        dev.DecodeLoop(*args, eviction=dev.DeviceEviction(other, 8))

    class Other:
        tokens = torch.zeros(6, dtype=torch.int32)
    with pytest.raises(ValueError, match="sampler's tokens"):
        dev.DecodeLoop(*args, logprobs=Other())
    loop = dev.DecodeLoop(*args, eviction=dev.DeviceEviction(attn, 8))
    assert len(loop._record) == 3
