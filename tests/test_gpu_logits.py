"""`mark_prompt_tokens` and `penalize_logits` through the C ABI against their definitions on the host in 64 bits.

Tolerance of the logits: every step rounds once in fp32, so err <= 2^-24 * (sum of the magnitudes of the step
results): |x1| for the product or quotient, then one for each of up to four additions and the product
frequency * count; 6 * 2^-24 * (|x1| + |frequency c| + |presence| + |bias|) covers them."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = float("inf")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _words(sets, vocab, width):
    rows = []
    for s in sets:
        w = [0] * width
        for i in s:
            w[i // 32] |= 1 << (i % 32)
        rows.append([x - (1 << 32) if x >= 1 << 31 else x for x in w])
    return torch.tensor(rows, dtype=torch.int32)


@pytest.mark.parametrize("vocab", [1, 31, 32, 33, 1024, 50257, 128256, 131073, 1 << 20])
@pytest.mark.parametrize("accumulate", [False, True])
def test_mark_prompt_tokens(vocab, accumulate):
    from paper_2502_02534_amd import binding as B
    rng = random.Random(vocab)
    lens = [0, 1, 2000, 300]
    tokens = [rng.choice([rng.randrange(vocab), rng.randrange(vocab), vocab - 1, 0]) for _ in range(sum(lens))]
    for i in range(5, 2000, 50):
        tokens[i] = rng.choice([-1, vocab, vocab + 7, -(1 << 31), (1 << 31) - 1])  # no tokens: ignored
    first = _starts(lens)
    width = -(-vocab // 32) + 3
    before = [set(rng.randrange(vocab) for _ in range(3)) for _ in lens]
    bits = _words(before, vocab, width)
    bits[:, -3:] = 12345  # words past the vocabulary are left alone
    want = [set(t for t in tokens[a:b] if 0 <= t < vocab) | (old if accumulate else set())
            for a, b, old in zip(first, first[1:], before)]
    dev = bits.to(DEV)
    print(f"mark vocab {vocab} accumulate {accumulate}", flush=True)
    B.mark_prompt_tokens(_i32(tokens), _i32(first), len(lens), vocab, dev, width, accumulate)
    torch.cuda.synchronize()
    expect = _words(want, vocab, width)
    expect[:, -3:] = 12345
    assert torch.equal(dev.cpu(), expect)


class Case:
    def __init__(self, rows, vocab, dtype="f32", seed=0, gen=40, pad=0, parts="rfpmtbg", by_step=False, prompts=2, grammars=3,
                 special=True):
        g = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        self.rows, self.vocab, self.dtype, self.pad = rows, vocab, dtype, pad
        t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.wide = (3 * torch.randn((rows, vocab + pad), generator=g)).to(t)
        x = self.wide[:, :vocab]
        if special and vocab > 40:
            x[:, 3], x[:, 4], x[:, 5], x[:, 6] = INF, -INF, 0.0, torch.finfo(t).min
            x[:, 7] = torch.finfo(t).max
            x[0, 9] = float("nan")
        width = -(-vocab // 32) + 1
        some = lambda k: {rng.randrange(vocab) for _ in range(k)}  # noqa: E731
        self.prompt_sets = [some(vocab // 5 + 1) for _ in range(prompts)] if "m" in parts else None
        self.prompt_of_row = [rng.randrange(-1, prompts) for _ in range(rows)]
        self.allowed_sets = [some(vocab // (2 + 3 * i) + 1) for i in range(grammars)] if "g" in parts else None
        if self.allowed_sets:
            self.allowed_sets[0] = set()  # a state that allows nothing
        self.allowed_of_row = [rng.randrange(-1, grammars) for _ in range(rows)]
        self.lens = [rng.choice([0, gen, rng.randrange(gen + 1)]) for _ in range(rows)]
        pick = lambda: rng.choice([rng.randrange(vocab), rng.randrange(min(vocab, 4)), -1, vocab])  # noqa: E731
        self.tokens = [[pick() for _ in range(gen)] for _ in range(rows)] if "t" in parts else None
        value = lambda lo, hi: lo + (hi - lo) * torch.rand(rows, generator=g)  # noqa: E731
        self.rep = value(0.7, 1.8) if "r" in parts else None
        self.freq = value(-0.5, 1.0) if "f" in parts else None
        self.pres = value(-0.5, 1.0) if "p" in parts else None
        self.biases = None
        if "b" in parts:
            self.biases = [[(i, rng.choice([rng.uniform(-5, 5), -100.0, torch.finfo(torch.float32).min, -INF, INF]))
                            for i in sorted(some(rng.choice([0, 1, min(vocab, 30)])) | {min(3, vocab - 1)})] + [(-1, 1.0), (vocab, 1.0)]
                           for _ in range(rows)]
        self.by_step, self.width = by_step, width

    def reference(self):
        x = self.wide[:, :self.vocab].double()
        mag = torch.zeros_like(x)
        for r in range(self.rows):
            count = torch.zeros(self.vocab, dtype=torch.float64)
            for t in (self.tokens[r][:self.lens[r]] if self.tokens else []):
                if 0 <= t < self.vocab:
                    count[t] += 1
            seen = count > 0
            if self.prompt_sets and self.prompt_of_row[r] >= 0:
                seen[list(self.prompt_sets[self.prompt_of_row[r]])] = True
            rho = float(self.rep[r]) if self.rep is not None else 1.0
            y = torch.where(seen, torch.where(x[r] > 0, x[r] / rho, x[r] * rho), x[r])
            f = (float(self.freq[r]) if self.freq is not None else 0.0) * count
            p = (float(self.pres[r]) if self.pres is not None else 0.0) * (count > 0)
            m = y.abs() + f.abs() + p.abs()
            y = torch.where(count > 0, y - f - p, y)
            if self.biases:
                for i, b in self.biases[r]:
                    if 0 <= i < self.vocab:
                        b = float(torch.tensor(b, dtype=torch.float32))
                        y[i] += b
                        m[i] += abs(b)
            if self.allowed_sets and self.allowed_of_row[r] >= 0:
                off = torch.ones(self.vocab, dtype=torch.bool)
                off[list(self.allowed_sets[self.allowed_of_row[r]])] = False
                y[off] = -INF
            x[r], mag[r] = y, m
        return x, mag

    def run(self, in_place=False, stream=None):
        from paper_2502_02534_amd import binding as B
        up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
        kw = dict(repetition=up(self.rep), frequency=up(self.freq), presence=up(self.pres))
        if self.prompt_sets:
            kw.update(prompt_bits=_words(self.prompt_sets, self.vocab, self.width).to(DEV), prompt_of_row=_i32(self.prompt_of_row))
        if self.allowed_sets:
            kw.update(allowed_bits=_words(self.allowed_sets, self.vocab, self.width).to(DEV), allowed_of_row=_i32(self.allowed_of_row))
        if self.tokens:
            tok = _i32(self.tokens)
            kw.update(tokens=tok.t().contiguous().t() if self.by_step else tok, token_lens=_i32(self.lens))
        if self.biases:
            flat = [e for row in self.biases for e in row]
            kw.update(bias_indptr=_i32(_starts([len(b) for b in self.biases])), bias_tokens=_i32([i for i, _ in flat]),
                      bias_values=torch.tensor([b for _, b in flat], dtype=torch.float32, device=DEV))
        pen = B.make_penalties(**kw)
        wide = self.wide.to(DEV)
        out = wide if in_place else torch.full((self.rows, self.vocab + 2 * self.pad), 9.0, device=DEV)
        torch.cuda.synchronize()
        B.penalize_logits(wide, B.SPD_F32 if self.dtype == "f32" else B.SPD_BF16, self.rows, self.vocab, wide.stride(0), pen, out,
                          out.stride(0), stream)
        torch.cuda.synchronize()
        assert in_place or bool((out[:, self.vocab:] == 9.0).all())
        if in_place:
            assert torch.equal(out[:, self.vocab:].cpu(), self.wide[:, self.vocab:])
        return out[:, :self.vocab].cpu()

    def check(self, **kw):
        print(f"logits {self.dtype} {self.rows} x {self.vocab}", flush=True)
        got = self.run(**kw).double()
        want, mag = self.reference()
        f32max = torch.finfo(torch.float32).max
        want = torch.where(want.abs() > f32max, torch.sign(want) * INF, want)  # past the range of fp32
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        fin = torch.isfinite(want)
        assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)])
        assert bool(((got - want).abs()[fin] <= 6 * 2.0 ** -24 * mag[fin]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 31, 32, 100, 1023, 4096, 4097, 8200, 50257])
def test_every_part_at_once(dtype, vocab):
    Case(5, vocab, dtype, seed=vocab).check()
    Case(3, vocab, dtype, seed=vocab + 1, pad=3, by_step=True, gen=700).check()


@pytest.mark.parametrize("parts", ["", "r", "rm", "rt", "f", "ft", "pt", "b", "g", "gb", "mtrfp"])
def test_parts_left_out(parts):
    Case(4, 5000, "f32", seed=len(parts), parts=parts).check()
    Case(4, 5001, "bf16", seed=len(parts) + 1, parts=parts).check()


@pytest.mark.parametrize("pad", [0, 1, 4, 5])
def test_in_place_and_strides(pad):
    Case(4, 3000, "f32", seed=pad, pad=pad).check(in_place=True)
    Case(4, 3001, "f32", seed=pad, pad=pad).check(in_place=True)
    Case(4, 3001, "bf16", seed=pad, pad=pad).check()
    Case(4, 3002, "f32", seed=pad, pad=pad).check(stream=torch.cuda.Stream())


def test_long_histories_and_one_token_repeated():
    c = Case(3, 9000, "f32", seed=1, gen=6000)
    c.check()
    c = Case(2, 9000, "bf16", seed=2, gen=5000)
    c.tokens = [[17] * 5000, [8999] * 5000]
    c.lens = [5000, 4999]
    c.check()


def test_lengths_beyond_the_stated_bound_are_cut_to_it():
    c = Case(2, 500, "f32", seed=4, gen=30)
    want = c.run()
    over = [x + (1000 if x == 30 else 0) for x in c.lens]
    c.lens, true = over, c.lens
    got = c.run()
    assert any(x == 30 for x in true)
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_many_rows_and_determinism():
    c = Case(300, 2000, "bf16", seed=7, gen=60)
    c.check()
    a, b = c.run(), c.run()
    assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def test_a_captured_call_follows_the_tokens():
    """One captured call, replayed while the history grows: a decode loop's use of it."""
    from paper_2502_02534_amd import binding as B
    rows, vocab = 4, 6000
    x = torch.randn((rows, vocab), device=DEV)
    tokens, lens = torch.zeros((10, rows), dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    freq = torch.full((rows,), 0.5, device=DEV)
    out = torch.empty_like(x)
    pen = B.make_penalties(frequency=freq, tokens=tokens.t(), token_lens=lens)
    call = lambda: B.penalize_logits(x, B.SPD_F32, rows, vocab, vocab, pen, out, vocab)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    want = x.clone()
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        tokens[step] = torch.tensor([5, 5, 5999, step], device=DEV)
        lens += 1
        counts = torch.zeros((rows, vocab), device=DEV)
        for t in range(step + 1):
            counts[torch.arange(rows, device=DEV), tokens[t].long()] += 1
        want = torch.where(counts > 0, x - 0.5 * counts - 0.0, x)


def test_marks_of_the_last_of_two_to_the_31_tokens():
    """Places of tokens that a thread would reach past 2^31 are not read."""
    from paper_2502_02534_amd import binding as B
    if torch.cuda.get_device_properties(0).total_memory < (24 << 30):
        pytest.skip("needs 9 GB of device memory")
    n, vocab = (1 << 31) - 1, 3000
    tokens = torch.empty(n, dtype=torch.int32, device=DEV)
    tail = torch.arange(100, dtype=torch.int32, device=DEV) * 29
    tokens[-100:] = tail
    indptr = torch.tensor([n - 100, n], dtype=torch.int32, device=DEV)
    bits = torch.zeros((1, 94), dtype=torch.int32, device=DEV)
    B.mark_prompt_tokens(tokens, indptr, 1, vocab, bits, 94)
    torch.cuda.synchronize()
    want = torch.zeros(94 * 32, dtype=torch.int64)
    want[tail.cpu().long()] = 1
    words = (want.view(94, 32) << torch.arange(32)).sum(1)
    assert torch.equal(bits[0].cpu().long() & 0xffffffff, words)
