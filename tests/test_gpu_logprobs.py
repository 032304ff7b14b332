"""`token_logprobs` through the C ABI against its definition in 64 bits, row by row.

Tolerances.  A row's exponents d = (x - max) / T carry three roundings, 3 * 2^-24 |d|, and the exponential a few units
of 2^-24 more; their sum's relative error is at most the mean of those over the row's probabilities, with a mean |d| of at most 20 here
below 4e-6, and its own fp32 partial sums (at most 2^8 additions one after another, then a tree) below 2^-16 / 4 = 4e-6.  So
  log p    err <= 8e-6 + 4e-7 |ref|   (its own d, |d| <= |ref| + ln Z, and two roundings)
  lse      err <= 8e-6 + 2e-7 |ref|
  entropy  err <= 2e-5 + 2e-6 ref     (sum p |d|: every term is off by as much as its exponential, and by its own d)
Tokens and ranks are equal."""
import math

import pytest

import readout_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LOWEST = torch.finfo(torch.float32).min


def call(x, temperature, tokens, top, outputs=None, stream=None, ws=None):
    from paper_2502_02534_amd import binding as B
    rows, vocab = x.shape
    f = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    i = lambda *s: torch.full(s, -7, dtype=torch.int32, device=DEV)  # noqa: E731
    o = {"logprobs": f(rows), "ranks": i(rows), "entropy": f(rows), "lse": f(rows), "top_tokens": i(rows, top), "top_logprobs": f(rows, top)}
    if outputs is not None:
        o = {k: v if k in outputs else None for k, v in o.items()}
    if top == 0:
        o["top_tokens"] = o["top_logprobs"] = None
    if ws is None:
        ws = torch.full((max(256, B.token_logprobs_workspace_size(rows, vocab, top)),), 0xA5, dtype=torch.uint8, device=DEV)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())  # (what was filled above)
    B.token_logprobs(x, B.SPD_BF16 if x.dtype == torch.bfloat16 else B.SPD_F32, rows, vocab, x.stride(0), temperature, tokens, top,
                     o["logprobs"], o["ranks"], o["entropy"], o["lse"], o["top_tokens"], o["top_logprobs"], ws, stream)
    return o


def near(got, ref, flat, slope, what):
    if math.isinf(ref):
        assert got == ref, (what, got, ref)
    else:
        assert abs(got - ref) <= flat + slope * abs(ref), (what, got, ref)


def check(x, temperature, tokens, top, rows=None, o=None):
    if o is None:
        o = call(x, temperature, tokens, top)
        torch.cuda.synchronize()
    o = {k: None if v is None else v.cpu() for k, v in o.items()}
    for r in range(x.shape[0]) if rows is None else rows:
        ref = R.logprobs(x[r].double().cpu(), 1.0 if temperature is None else float(temperature[r]), int(tokens[r]) if tokens is not None else -1, top)
        if o["logprobs"] is not None:
            near(float(o["logprobs"][r]), ref["logprob"], 8e-6, 4e-7, ("logprob", r))
        if o["ranks"] is not None:
            assert int(o["ranks"][r]) == ref["rank"], r
        if o["entropy"] is not None:
            near(float(o["entropy"][r]), ref["entropy"], 2e-5, 2e-6, ("entropy", r))
        if o["lse"] is not None:
            near(float(o["lse"][r]), ref["lse"], 8e-6, 2e-7, ("lse", r))
        if top and o["top_tokens"] is not None:
            assert o["top_tokens"][r].tolist() == ref["top_tokens"], r
        if top and o["top_logprobs"] is not None:
            for got, want in zip(o["top_logprobs"][r].tolist(), ref["top_logprobs"]):
                near(got, want, 8e-6, 4e-7, ("top", r))


def logits(rows, vocab, dtype, seed=0, pad=0, sigma=3.0, first=0):
    """Rows `pad` elements apart, the first `first` elements into the memory; what lies between them is NaN."""
    g = torch.Generator().manual_seed(seed)
    wide = torch.full((rows * (vocab + pad) + first,), float("nan"))
    view = wide[first:].view(rows, vocab + pad)[:, :vocab]
    view.copy_(torch.randn(rows, vocab, generator=g) * sigma)
    return wide.to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)[first:].view(rows, vocab + pad)[:, :vocab]


def some_tokens(rows, vocab, seed=0):
    return torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(seed + 99)).to(torch.int32).to(DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 63, 64, 65, 255, 256, 1000, 1024, 4097, 16383, 16384, 16385, 32000, 50257, 128256])
def test_sizes(dtype, vocab):
    rows = 5 if vocab <= 4097 else 3
    x = logits(rows, vocab, dtype, seed=vocab)
    t = torch.tensor([1.0, 0.2, 0.0, 1.7, 0.7][:rows], device=DEV)
    check(x, t, some_tokens(rows, vocab), min(vocab, 20))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,first", [(0, 0), (1, 0), (8, 0), (5, 3), (0, 1), (63, 7)])
@pytest.mark.parametrize("vocab", [1023, 20001])
def test_strides_and_starts(dtype, pad, first, vocab):
    x = logits(4, vocab, dtype, seed=pad, pad=pad, first=first)
    check(x, None, some_tokens(4, vocab), 7)


@pytest.mark.parametrize("rows", [1, 17, 130, 300, 700, 2100])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(rows, dtype):
    x = logits(rows, 2000, dtype, seed=rows)
    t = 0.3 + torch.rand(rows, generator=torch.Generator().manual_seed(rows)).to(DEV)
    check(x, t, some_tokens(rows, 2000), 5, rows=sorted({0, 1, rows // 2, rows - 2, rows - 1} & set(range(rows))))


@pytest.mark.parametrize("top", [0, 1, 2, 5, 20, 63, 64])
@pytest.mark.parametrize("rows,vocab", [(3, 64), (3, 5000), (2, 128256), (600, 128)])
def test_number_of_alternatives(top, rows, vocab):
    x = logits(rows, vocab, "f32", seed=top)
    check(x, None, some_tokens(rows, vocab), top, rows=range(min(rows, 3)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 16384, 40000])
def test_ties_and_orders(dtype, vocab):
    """Equal logits everywhere, few different ones, rising, falling, the largest at the end, in one stretch."""
    i = torch.arange(vocab, dtype=torch.float32)
    few = torch.randint(-2, 3, (vocab,), generator=torch.Generator().manual_seed(1)).float()
    stretch = -i % 7 * 0.5
    stretch[vocab // 3:vocab // 3 + 64] += 9.0
    end = torch.zeros(vocab)
    end[-1] = 20.0
    stride = torch.zeros(vocab)
    stride[5::256] = 8.0
    signed_zero = torch.where(i % 2 == 0, 0.0, -0.0)
    x = torch.stack([torch.zeros(vocab), few, i / vocab * 30, -i / vocab * 30, end, stretch, stride, signed_zero])
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
    for top in (1, 20, 64):
        check(x, None, some_tokens(len(x), vocab, top), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [100, 20000, 70000])
def test_masked_tokens(dtype, vocab):
    """-inf everywhere, everywhere but for a few tokens, in front, behind; the type's lowest value in their place."""
    base = torch.randn(vocab, generator=torch.Generator().manual_seed(2)) * 3
    rows = []
    for low in (-math.inf, LOWEST if dtype == "f32" else torch.finfo(torch.bfloat16).min):
        one = torch.full((vocab,), low)
        one[vocab // 2] = 1.5
        few = torch.full((vocab,), low)
        few[::vocab // 9] = base[::vocab // 9]
        front, back = base.clone(), base.clone()
        front[: vocab - 30] = low
        back[30:] = low
        rows += [torch.full((vocab,), low), one, few, front, back]
    x = torch.stack(rows).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
    tokens = torch.tensor([0, vocab // 2, 1, 0, vocab - 1] * 2, dtype=torch.int32, device=DEV)
    o = call(x, None, tokens, 40)
    for r in range(len(x)):
        if not torch.isfinite(x[r].max()):
            assert float(o["lse"][r]) == -math.inf and float(o["entropy"][r]) == 0.0 and float(o["logprobs"][r]) == -math.inf
            assert o["top_tokens"][r].tolist() == list(range(40))
            assert torch.isneginf(o["top_logprobs"][r]).all()
    # (log p of tokens at the lowest value beside others: the plain form's difference overflows to the same)
    keep = [r for r in range(len(x))]
    o = {k: v[keep] for k, v in o.items()}
    want = x[keep].double().cpu()
    for r in range(len(keep)):
        ref = R.logprobs(want[r], 1.0, int(tokens[r]), 40)
        assert int(o["ranks"][r]) == ref["rank"] and o["top_tokens"][r].tolist() == ref["top_tokens"]
        near(float(o["entropy"][r]), ref["entropy"], 2e-5, 2e-6, r)
        near(float(o["logprobs"][r]), ref["logprob"], 8e-6, 4e-7, r)
        for got, exact in zip(o["top_logprobs"][r].tolist(), ref["top_logprobs"]):
            near(got, exact, 8e-6, 4e-7, r)


def test_lowest_values_with_a_temperature():
    """(x - max) / T of a row of the lowest value is 0, not inf - inf; its lse overflows."""
    x = torch.full((2, 5000), LOWEST, device=DEV)
    o = call(x, torch.tensor([0.2, 0.5], device=DEV), some_tokens(2, 5000), 3)
    for r in range(2):
        assert abs(float(o["logprobs"][r]) + math.log(5000)) < 8e-6 and abs(float(o["entropy"][r]) - math.log(5000)) < 2e-5
        assert float(o["lse"][r]) == -math.inf and o["top_tokens"][r].tolist() == [0, 1, 2]


def test_tokens_outside_the_vocabulary():
    x = logits(6, 777, "f32")
    tokens = torch.tensor([-1, 777, 776, 0, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    check(x, None, tokens, 2)


@pytest.mark.parametrize("outputs", [("logprobs",), ("ranks",), ("entropy",), ("lse",), ("top_tokens",), ("top_logprobs",),
                                     ("logprobs", "top_tokens", "top_logprobs")])
@pytest.mark.parametrize("rows,vocab", [(3, 30000), (500, 3000)])
def test_outputs_left_out(outputs, rows, vocab):
    x = logits(rows, vocab, "bf16")
    tokens = some_tokens(rows, vocab)
    check(x, None, tokens, 4, rows=range(3), o=call(x, None, tokens if set(outputs) & {"logprobs", "ranks"} else None, 4, outputs))


def test_nan_logits_end():
    """Results are the caller's own, but the call returns, and other rows have theirs."""
    x = logits(5, 40000, "f32")
    x[1] = float("nan")
    x[2, ::3] = float("nan")
    x[3, 7] = float("inf")
    tokens = some_tokens(5, 40000)
    o = call(x, None, tokens, 64)
    torch.cuda.synchronize()
    top = o["top_tokens"]
    assert int(top.min()) >= -7 and int(top.max()) < 40000
    check(x[:1], None, tokens[:1], 64, o={k: v[:1] for k, v in o.items()})
    check(x[4:], None, tokens[4:], 64, o={k: v[4:] for k, v in o.items()})


@pytest.mark.parametrize("rows,vocab", [(2, 128256), (400, 5000)])
def test_calls_repeat_to_the_bit_and_replay(rows, vocab):
    """The same answer every time, on another stream, and from a captured graph with eager work between its replays."""
    from paper_2502_02534_amd import binding as B
    x = logits(rows, vocab, "bf16", seed=5)
    tokens = some_tokens(rows, vocab)
    first = call(x, None, tokens, 20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(x, None, tokens, 20)
    torch.cuda.current_stream().wait_stream(side)
    third = call(x, None, tokens, 20, stream=side)
    torch.cuda.synchronize()
    for k in first:
        assert torch.equal(first[k], second[k]) and torch.equal(first[k], third[k]), k
    ws = torch.empty(max(256, B.token_logprobs_workspace_size(rows, vocab, 20)), dtype=torch.uint8, device=DEV)
    call(x, None, tokens, 20, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = call(x, None, tokens, 20, ws=ws)
    other = logits(rows, vocab, "bf16", seed=6)
    x0 = x.clone()
    for n in range(4):
        x.copy_(other if n % 2 else x0)
        graph.replay()
        torch.cuda.synchronize()
        eager = call(x, None, tokens, 20)
        torch.cuda.synchronize()
        for k in o:
            assert torch.equal(o[k], eager[k]), (n, k)


def test_given_tokens_of_far_rows():
    """Rows past 2^31 elements."""
    rows, vocab = 3, 1000
    stride = 1 << 30
    wide = torch.empty((rows - 1) * stride + vocab, dtype=torch.bfloat16, device=DEV)
    x = wide.as_strided((rows, vocab), (stride, 1))
    x.copy_(logits(rows, vocab, "bf16", seed=8))
    check(x, None, some_tokens(rows, vocab), 5)
