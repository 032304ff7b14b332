"""`select_kv_tokens` and `compact_kv` through the C ABI against their definitions.  Both move and order what is given: everything is equal."""
import pytest

import readout_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PAGE = 16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def select(weights, lens, budgets, max_new, sinks, recent, max_kv=None, source=None, stream=None, ws=None):
    from paper_2502_02534_amd import binding as B
    n, heads, stride = weights.shape
    mk = stride if max_kv is None else max_kv
    if source is None:
        source = torch.full((n, heads, max(1, min(max_new, mk)) + 3), -5, dtype=torch.int32, device=DEV)
    new = torch.full((n,), -5, dtype=torch.int32, device=DEV)
    if ws is None:
        ws = torch.full((max(256, B.select_kv_tokens_workspace_size(n, heads, mk)),), 0xA5, dtype=torch.uint8, device=DEV)
    B.select_kv_tokens(weights, stride, n, heads, lens, mk, budgets, max_new, sinks, recent, source, source.stride(1), new, ws, stream)
    return source, new


def check_select(weights, lens, budgets, sinks, recent, max_new=None):
    most = max(1, max(budgets)) if max_new is None else max_new
    source, new = select(weights.to(DEV), i32(lens), None if budgets is None else i32(budgets), most, sinks, recent)
    torch.cuda.synchronize()
    source, new = source.cpu(), new.cpu()
    for b, n in enumerate(lens):
        budget = most if budgets is None else min(most, max(0, budgets[b]))
        n = max(0, min(n, weights.shape[2]))
        assert int(new[b]) == min(n, budget)
        for j in range(weights.shape[1]):
            want = R.kept(weights[b, j].tolist(), n, budget, sinks, recent)
            assert source[b, j, :len(want)].tolist() == want, (b, j, n, budget)
            assert (source[b, j, len(want):] == -5).all()


def draw(n, heads, stride, seed, kind="heavy"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, stride, generator=g)
    if kind == "heavy":
        return torch.exp(3 * x)
    if kind == "signed":
        return x
    return torch.randint(0, 4, x.shape, generator=g).float() - 1.0  # ties


@pytest.mark.parametrize("kind", ["heavy", "signed", "ties"])
@pytest.mark.parametrize("length", [1, 2, 63, 64, 65, 200, 255, 256, 257, 511, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 5000, 9000, 16384, 20001])
def test_lengths(kind, length):
    w = draw(1, 2, length + 2, length, kind)
    for budget in sorted({1, length // 2, length - 1, length} - {0}):
        check_select(w, [length], [budget], 4, 16)


@pytest.mark.parametrize("sinks,recent", [(0, 0), (4, 0), (0, 64), (4, 64), (500, 500), (1, 10 ** 9), (10 ** 9, 1), (0, 7)])
def test_sinks_and_recent(sinks, recent):
    lens = [0, 1, 5, 63, 64, 65, 128, 300, 700, 701]
    w = draw(len(lens), 2, 701, 3)
    for budget in (0, 1, 2, 10, 64, 100, 300, 699, 700, 5000):
        check_select(w, lens, [budget] * len(lens), sinks, recent, max_new=701)


def test_budgets_of_their_own():
    lens = [300, 40, 0, 257, 300, 300, 100]
    w = draw(7, 3, 300, 4)
    check_select(w, lens, [100, 100, 100, 256, -3, 0, 99], 2, 8)
    check_select(w, lens, None, 2, 8, max_new=77)
    check_select(w, lens, [500] * 7, 2, 8, max_new=150)          # budgets above the bound count as it


@pytest.mark.parametrize("length", [100, 1500, 12000, 70000])
def test_equal_zero_infinite_and_missing_weights(length):
    x = torch.zeros(6, 1, length)
    x[1, 0, ::2] = -0.0                                            # both zeros are equal
    x[2] = float("inf")
    x[3] = float("nan")
    x[4, 0, ::3] = float("nan")
    x[4, 0, 1::3] = float("-inf")
    x[5, 0] = torch.arange(length).float() * 1e-40                 # numbers below the normal ones
    check_select(x, [length] * 6, [length // 3] * 6, 4, 16)


def test_lengths_past_the_bound():
    w = draw(3, 2, 120, 5)
    source, new = select(w.to(DEV), i32([500, 120, -4]), None, 60, 0, 4, max_kv=100)
    for b, n in enumerate((100, 100, 0)):
        for j in range(2):
            want = R.kept(w[b, j].tolist(), n, 60, 0, 4)
            assert source[b, j, :len(want)].tolist() == want
    assert new.tolist() == [60, 60, 0]


@pytest.mark.parametrize("length", [70000, 150001])
def test_long_rows(length):
    check_select(draw(1, 2, length, 6), [length], [length // 7], 4, 64)
    check_select(draw(1, 1, length, 7, "ties"), [length], [length - 3], 0, 0)


def test_many_rows():
    lens = [(53 * i) % 130 for i in range(400)]
    check_select(draw(400, 4, 130, 8, "ties"), lens, [50] * 400, 1, 8)


# ---- compaction ------------------------------------------------------------------------------------------------

class Cache:
    """Sequences of `lens` tokens with `room` more each."""

    def __init__(self, dtype, hkv, d, lens, page, seed=0, room=0, stride_pad=0, kv_pad=0, pages_between=2):
        g = torch.Generator().manual_seed(seed)
        t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.dtype, self.hkv, self.d, self.lens, self.page = dtype, hkv, d, lens, page
        if page:
            held = [-(-(n + room) // PAGE) for n in lens]
            self.indptr = torch.tensor([0] + held).cumsum(0).to(torch.int32)
            pool = sum(held) + pages_between
            self.pages = torch.randperm(max(pool, 1), generator=g)[: max(1, sum(held))].to(torch.int32)
            shape = (max(pool, 1), hkv, PAGE, d)
        else:
            self.indptr, self.pages = torch.tensor([0] + [n + room for n in lens]).cumsum(0).to(torch.int32), None
            shape = (max(1, int(self.indptr[-1])), hkv * d + kv_pad)
        self.kv_pad = kv_pad
        self.k, self.v = torch.randn(shape, generator=g).to(t), torch.randn(shape, generator=g).to(t)
        self.weights = torch.rand(len(lens), hkv, max(max(lens), 1) + stride_pad, generator=g)

    def heads(self, x):
        return x if self.page else x[:, : self.hkv * self.d].unflatten(1, (self.hkv, self.d))

    def desc(self):
        from paper_2502_02534_amd import binding as B
        return B.make_prompt_desc(dtype=B.SPD_F32 if self.dtype == "f32" else B.SPD_BF16, num_q_heads=self.hkv, num_kv_heads=self.hkv,
                                  head_dim=self.d, num_prompts=len(self.lens), page_size=self.page,
                                  kv_stride=self.hkv * self.d + self.kv_pad if self.kv_pad else 0)


def expected(old, new, sources, weights, weights_out):
    """What the pools and weights hold afterwards.  sources[b][j]: tokens of places 0, 1, ..."""
    k, v, w = new.k.clone(), new.v.clone(), weights_out.clone()
    for b in range(len(old.lens)):
        for j in range(old.hkv):
            for i, src in enumerate(sources[b][j]):
                to, at = R.slots(new.indptr, new.pages, b, i), R.slots(old.indptr, old.pages, b, src)
                R.row(new.heads(k), to, j).copy_(R.row(old.heads(old.k), at, j))
                R.row(new.heads(v), to, j).copy_(R.row(old.heads(old.v), at, j))
                w[b, j, i] = weights[b, j, src]
            w[b, j, len(sources[b][j]):] = 0
    return k, v, w


def run_compact(old, new, sources, max_new=None, in_place=True, head_shared=False, weights=True, weights_in_place=True, stream=None):
    from paper_2502_02534_amd import binding as B
    n, hkv = len(old.lens), old.hkv
    most = max([1] + [len(s) for x in sources for s in x]) if max_new is None else max_new
    table = torch.full((n, 1 if head_shared else hkv, most + 2), 2 ** 31 - 1, dtype=torch.int32)
    for b in range(n):
        for j in range(table.shape[1]):
            table[b, j, :len(sources[b][j])] = torch.tensor(sources[b][j], dtype=torch.int32)
    table = table.to(DEV)
    new_lens = i32([len(x[0]) for x in sources])
    up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
    ki, kp, k, v = up(old.indptr), up(old.pages), up(old.k), up(old.v)
    oi, op, ko, vo = (ki, kp, k, v) if in_place else (up(new.indptr), up(new.pages), up(new.k), up(new.v))
    w = up(old.weights) if weights else None
    wo = None if w is None else w if weights_in_place else torch.full_like(w, 7.0)
    lens = torch.full((n,), -9, dtype=torch.int32, device=DEV)
    B.compact_kv(old.desc(), table, table.stride(0), 0 if head_shared else table.stride(1), new_lens, most, ki, kp, k, v, oi, op, ko, vo, w, wo,
                 0 if w is None else w.stride(1), lens, stream)
    torch.cuda.synchronize()
    assert torch.equal(lens, new_lens)
    if not in_place:
        assert torch.equal(k.cpu(), old.k) and torch.equal(v.cpu(), old.v)
    return ko.cpu(), vo.cpu(), None if wo is None else wo.cpu()


def same(a, b):
    return torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a.view(torch.int32),
                       b.view(torch.int16) if b.dtype == torch.bfloat16 else b.view(torch.int32))


def lists(cache, budget, sinks, recent, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [[R.kept(torch.rand(max(n, 1), generator=g).tolist(), n, budget, sinks, recent) for _ in range(cache.hkv)] for n in cache.lens]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 64, 80, 128, 256])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("budget,recent", [(100, 0), (100, 30), (290, 64), (1, 0), (0, 0), (1000, 4)])
def test_in_place(dtype, d, page, budget, recent):
    """Gaps filled from behind, and the last tokens shifted over places that they are read from."""
    c = Cache(dtype, 2, d, [300, 0, 1, 101, 100, 17], page, seed=d)
    s = lists(c, budget, 2, recent)
    k, v, w = run_compact(c, c, s)
    ek, ev, ew = expected(c, c, s, c.weights, c.weights)
    assert same(k, ek) and same(v, ev) and torch.equal(w, ew)


@pytest.mark.parametrize("page", [0, 16])
def test_in_order(page):
    """Any list of sources that are not below their places: here the tokens that stay, in their order."""
    c = Cache("bf16", 3, 128, [700, 333], page, room=20, kv_pad=0 if page else 8)
    g = torch.Generator().manual_seed(1)
    s = [[sorted(torch.randperm(n, generator=g)[: n // 2].tolist()) for _ in range(3)] for n in c.lens]
    s = [[x[: min(map(len, y))] for x in y] for y in s]
    k, v, w = run_compact(c, c, s)
    ek, ev, ew = expected(c, c, s, c.weights, c.weights)
    assert same(k, ek) and same(v, ev) and torch.equal(w, ew)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("page", [0, 16])
def test_into_other_pages(dtype, d, page):
    old = Cache(dtype, 2, d, [300, 0, 40, 513], page, seed=1)
    new = Cache(dtype, 2, d, [120, 3, 40, 120], page, seed=2)
    s = lists(old, 120, 4, 20)
    k, v, w = run_compact(old, new, s, in_place=False, weights_in_place=False)
    ek, ev, ew = expected(old, new, s, old.weights, torch.full_like(old.weights, 7.0))
    assert same(k, ek) and same(v, ev) and torch.equal(w, ew)


def test_one_pool_two_tables():
    """The pages of a prompt that others still read stay as they are."""
    from paper_2502_02534_amd import binding as B
    g = torch.Generator().manual_seed(3)
    pool = torch.randn(20, 2, PAGE, 64, generator=g).to(torch.bfloat16)
    s = i32([[[0, 50, 2, 60, 99], [1, 50, 2, 70, 98]]])
    k, v = pool.to(DEV), (pool * 2).to(DEV)
    before = k.clone()
    old, new = i32([9, 3, 17, 4, 5, 6, 7]), i32([12])
    B.compact_kv(B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=2, num_kv_heads=2, head_dim=64, num_prompts=1, page_size=16), s, s.stride(0),
                 s.stride(1), i32([5]), 5, i32([0, 7]), old, k, v, i32([0, 1]), new, k, v, None, None, 0, None)
    for j in range(2):
        for i in range(5):
            t = int(s[0, j, i])
            assert torch.equal(k[12, j, i], before[int(old[t // PAGE]), j, t % PAGE])
    keep = [p for p in range(20) if p != 12]
    assert torch.equal(k[keep], before[keep]) and torch.equal(k[12, :, 5:], before[12, :, 5:])


@pytest.mark.parametrize("page", [0, 16])
def test_one_list_for_all_heads_and_no_weights(page):
    c = Cache("bf16", 4, 64, [200, 90], page)
    one = [R.kept(torch.rand(n, generator=torch.Generator().manual_seed(n)).tolist(), n, 70, 0, 5) for n in c.lens]
    s = [[x] * 4 for x in one]
    k, v, w = run_compact(c, c, s, head_shared=True)
    ek, ev, ew = expected(c, c, s, c.weights, c.weights)
    assert same(k, ek) and same(v, ev) and torch.equal(w, ew)
    k, v, w = run_compact(c, c, s, weights=False)
    assert same(k, ek) and same(v, ev) and w is None


def test_places_that_stay():
    """Sources below their place, past the sequence's table or the bound are left alone; lengths past the bound count as it."""
    from paper_2502_02534_amd import binding as B
    c = Cache("f32", 1, 64, [64, 64], 16, pages_between=0)
    k, v, w = c.k.to(DEV), c.v.to(DEV), c.weights.to(DEV)
    s = i32([[[3, 0, 64, 2 ** 31 - 1, 63, -1, 10 ** 6, 7, 9]], [[0, 1, 2, 3, 4, 5, 6, 7, 60]]])
    ki, pages, lens = c.indptr.to(DEV), c.pages.to(DEV), i32([0, 0])
    B.compact_kv(c.desc(), s, s.stride(0), s.stride(1), i32([8, 10 ** 6]), 9, ki, pages, k, v, ki, pages, k, v, w, w, 64, lens)
    assert lens.tolist() == [8, 9]
    at = lambda b, t: (int(c.pages[int(c.indptr[b]) + t // PAGE]), 0, t % PAGE)  # noqa: E731
    want = c.k.clone()
    for b, moves in ((0, {0: 3, 4: 63}), (1, {8: 60})):
        for to, src in moves.items():
            want[at(b, to)] = c.k[at(b, src)]
    assert torch.equal(k.cpu(), want)
    ew = c.weights.clone()
    ew[0, 0, 0], ew[0, 0, 4], ew[1, 0, 8] = ew[0, 0, 3], ew[0, 0, 63], ew[1, 0, 60]
    ew[0, 0, 2] = ew[0, 0, 3] = ew[0, 0, 6] = 0          # (their sources lie past the row of weights)
    ew[0, 0, 8:], ew[1, 0, 9:] = 0, 0
    assert torch.equal(w.cpu(), ew)


def test_shifts_of_long_rows():
    """A shift by one, by a few and by many places over thousands of tokens, where every place is read after its neighbour was written."""
    for d, shift, n in ((128, 1, 3000), (64, 5, 2500), (256, 300, 2000), (128, 16, 2048)):
        c = Cache("bf16", 2, d, [n, n - 7], 16, seed=shift)
        s = [[list(range(shift, x)) for _ in range(2)] for x in c.lens]
        s = [[x[: n - shift - 7] for x in y] for y in s]
        k, v, w = run_compact(c, c, s)
        ek, ev, ew = expected(c, c, s, c.weights, c.weights)
        assert same(k, ek) and same(v, ev) and torch.equal(w, ew)


def test_select_and_compact_replay():
    """Both in one graph, with eager work between the replays."""
    from paper_2502_02534_amd import binding as B
    c = Cache("bf16", 2, 64, [500, 260], 16)
    k0, v0, w0 = c.k.to(DEV), c.v.to(DEV), c.weights.to(DEV)
    k, v, w = k0.clone(), v0.clone(), w0.clone()
    lens, ki, pages = i32(c.lens), c.indptr.to(DEV), c.pages.to(DEV)
    source = torch.zeros((2, 2, 100), dtype=torch.int32, device=DEV)
    new, lens_out = i32([0, 0]), i32([0, 0])
    ws = torch.empty(max(256, B.select_kv_tokens_workspace_size(2, 2, 500)), dtype=torch.uint8, device=DEV)

    def step():
        B.select_kv_tokens(w, w.stride(1), 2, 2, lens, 500, None, 100, 4, 16, source, 100, new, ws)
        B.compact_kv(c.desc(), source, 200, 100, new, 100, ki, pages, k, v, ki, pages, k, v, w, w, w.stride(1), lens_out)

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (k, v, w, lens_out, source)]
    s = [[R.kept(c.weights[b, j].tolist(), n, 100, 4, 16) for j in range(2)] for b, n in enumerate(c.lens)]
    ek, ev, ew = expected(c, c, s, c.weights, c.weights)
    assert same(k.cpu(), ek) and same(v.cpu(), ev) and torch.equal(w.cpu(), ew)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for x, y in ((k, k0), (v, v0), (w, w0)):
            x.copy_(y)
        source.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((k, v, w, lens_out, source), want):
            assert torch.equal(x, y)


def test_far_pages():
    """Rows past 2^31 elements."""
    from paper_2502_02534_amd import binding as B
    pages = 2 ** 31 // (PAGE * 64) + 40
    k = torch.zeros((pages, 1, PAGE, 64), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    table = i32([pages - 1, pages - 20, pages - 3])
    g = torch.Generator(device=DEV).manual_seed(1)
    for x in (k, v):
        x[table.long()] = torch.randn((3, 1, PAGE, 64), generator=g, device=DEV).to(torch.bfloat16)
    kw, vw = (x[table.long()].transpose(1, 2).reshape(48, 64).clone() for x in (k, v))
    s = list(range(10)) + [40, 47]
    starts = i32([0, 3])
    B.compact_kv(B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=1, num_kv_heads=1, head_dim=64, num_prompts=1, page_size=16), i32(s), 12, 12,
                 i32([12]), 12, starts, table, k, v, starts, table, k, v, None, None, 0, None)
    for x, y in ((k, kw), (v, vw)):
        assert torch.equal(x[table.long()].transpose(1, 2).reshape(48, 64)[:12], y[s])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("budget,recent", [(1500, 0), (1023, 64), (1500, 1490), (2890, 20)])
def test_long_rows_in_place(dtype, page, budget, recent):
    """Few long rows: some whose gaps are filled from behind the new length, in any order, beside some that read places which others
    write."""
    c = Cache(dtype, 2, 64, [3000, 2900, 1024, 40, 0], page, seed=budget)
    s = lists(c, budget, 4, recent)
    k, v, w = run_compact(c, c, s)
    ek, ev, ew = expected(c, c, s, c.weights, c.weights)
    assert same(k, ek) and same(v, ev) and torch.equal(w, ew)


@pytest.mark.parametrize("length", [2040, 5000, 32768])
def test_signs_infinities_and_missing_weights_together(length):
    """A row's lowest key and its highest lie as far apart as any two, beside places that hold no token."""
    x = draw(2, 2, length, length, "signed")
    x[0, :, 7::11], x[0, 0, 5::13] = float("nan"), float("-inf")
    x[1, 0, 3::17] = float("inf")
    x[1, 1] = torch.randint(0, 3, (length,), generator=torch.Generator().manual_seed(1)).float() - 1.0
    for budget in (length // 20, length // 2, length - 70):
        check_select(x, [length, length - 333], [budget] * 2, 4, 60)
