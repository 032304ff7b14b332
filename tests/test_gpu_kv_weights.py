"""`accumulate_kv_weights` through the C ABI against its definition in 64 bits.

Tolerance.  With M the largest scale * sum_c |q_c k_c| of a sequence, a score is off by a few units of 2^-24 M and its exponent by as
many of 2^-24 |lse| (|lse| <= 60 here), which is the relative error of a term: 1e-5 max(1, M / 60) allows three.  The terms are positive, so
their sum (fp32: at most 2^10 one after another and a tree of partial sums, each 2^-24 of what it has) has it too: 3e-5 max(1, M / 60) of the
result, and 1e-30 for results near zero."""
import math

import pytest

import readout_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PAGE = 16


class Problem:
    def __init__(self, dtype, hq, hkv, d, queries, kv, page=0, causal=False, seed=0, decay=1.0, old=True, spare=0, stride_pad=0,
                 lead=0, strides=False, scale=0.0, elsewhere=0.0, peak=1.0):
        from paper_2502_02534_amd import binding as B
        g = torch.Generator().manual_seed(seed)
        t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.hq, self.hkv, self.d, self.page, self.causal, self.decay, self.kv = hq, hkv, d, page, causal, decay, kv
        self.total = lead + sum(queries) + spare
        self.query_indptr = torch.tensor([lead] + queries).cumsum(0).to(torch.int32)
        self.kv_lens = torch.tensor(kv, dtype=torch.int32)
        q = (torch.randn(max(self.total, 1), hq * d + (16 if strides else 0), generator=g) * peak).to(t)
        self.q = q[:, : hq * d].unflatten(1, (hq, d))
        if page:
            held = [-(-n // PAGE) for n in kv]
            pool = sum(held) + 3
            self.kv_indptr = torch.tensor([0] + held).cumsum(0).to(torch.int32)
            self.pages = torch.randperm(pool, generator=g)[: max(1, sum(held))].to(torch.int32)
            self.k = torch.randn(pool, hkv, PAGE, d, generator=g).to(t)
            live = torch.zeros(pool, PAGE, dtype=torch.bool)
            for b, n in enumerate(kv):
                for at in range(n):
                    live[self.pages[self.kv_indptr[b] + at // PAGE], at % PAGE] = True
            self.k[~live[:, None, :, None].expand_as(self.k)] = float("nan")
        else:
            self.kv_indptr, self.pages = torch.tensor([0] + kv).cumsum(0).to(torch.int32), None
            k = torch.randn(max(1, sum(kv)), hkv * d + (16 if strides else 0), generator=g).to(t)
            self.k = k[:, : hkv * d].unflatten(1, (hkv, d))
        self.scale = scale if scale else 1 / math.sqrt(d)
        self.stride = max(kv) + stride_pad
        shape = (len(kv), hkv, self.stride)
        self.old = torch.rand(shape, generator=g) * 3 if old else None
        self.out = torch.randn(shape, generator=g)
        self.desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=hq, num_kv_heads=hkv, head_dim=d,
                                       num_prompts=len(kv), page_size=page, causal=causal, sm_scale=scale,
                                       q_stride=self.q.stride(0) if strides else 0, kv_stride=self.k.stride(0) if strides and not page else 0)
        self.max_query, self.max_kv = max(queries), max(kv)
        # the queries' log-sum-exp over what they see here (and `elsewhere`)
        grp = hq // hkv
        self.lse = torch.full((max(self.total, 1), hq), float("nan"))
        for b, n in enumerate(queries):
            q0 = int(self.query_indptr[b])
            for i in range(n):
                see = max(0, min(kv[b], kv[b] - n + i + 1)) if causal else kv[b]
                for h in range(hq):
                    if see == 0:
                        self.lse[q0 + i, h] = -math.inf if not elsewhere else elsewhere
                        continue
                    k = self.keys(b, h // grp)[:see].double()
                    s = k @ self.q[q0 + i, h].double() * self.scale
                    x = torch.logsumexp(s, 0)
                    self.lse[q0 + i, h] = float(torch.logaddexp(x, torch.tensor(elsewhere, dtype=torch.float64))) if elsewhere else float(x)

    def keys(self, b, j):
        n, at = self.kv[b], int(self.kv_indptr[b])
        if self.page:
            return self.k[self.pages[at:at + -(-n // PAGE)].long()].transpose(1, 2).flatten(0, 1)[:n, j]
        return self.k[at:at + n, j]

    def up(self):
        up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
        # (a view's strides survive as the whole tensor's copy)
        whole = lambda x: x._base.to(DEV)[..., : x.shape[1] * x.shape[2]].unflatten(1, x.shape[1:]) if x._base is not None else x.to(DEV)  # noqa: E731
        return dict(q=whole(self.q), k=self.k.to(DEV) if self.page else whole(self.k), qi=up(self.query_indptr), kl=up(self.kv_lens),
                    ki=up(self.kv_indptr), pages=up(self.pages), lse=up(self.lse), old=up(self.old), out=up(self.out))

    def launch(self, s, stream=None, ws=None, max_query=None, max_kv=None):
        from paper_2502_02534_amd import binding as B
        mq, mk = max_query or self.max_query, max_kv or self.max_kv
        size = B.accumulate_kv_weights_workspace_size(self.desc, self.total, mq, mk)
        if ws is None:
            ws = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device=DEV)  # (NaN)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())  # (what was filled above)
        B.accumulate_kv_weights(self.desc, s["q"], s["k"], s["qi"], s["kl"], s["ki"], s["pages"], s["lse"], self.total, mq, mk, self.decay,
                                s["old"], s["out"], s["out"].stride(1), ws, stream)
        return s["out"]

    def reference(self):
        return R.weights(self.q, lambda b, t, j: self.keys(b, j)[t], self.query_indptr, self.kv_lens, self.lse, self.causal, self.scale,
                         self.decay, self.old, self.out, self.hkv)

    def check(self, got=None):
        if got is None:
            got = self.launch(self.up())
            torch.cuda.synchronize()
        ref, size = self.reference()
        got = got.double().cpu()
        tol = 3e-5 * (size / 60).clamp(min=1.0)[:, None, None] * ref.abs() + 1e-30
        for b, n in enumerate(self.kv):
            err = (got[b, :, :n] - ref[b, :, :n]).abs()
            assert bool((err <= tol[b, :, :n]).all()), (b, float((err / tol[b, :, :n]).max()))
            assert torch.equal(got[b, :, n:], ref[b, :, n:]), "places without a token were written"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (8, 2, 128), (3, 3, 80), (2, 1, 256), (16, 1, 96), (6, 2, 8), (5, 1, 248), (40, 2, 128)])
@pytest.mark.parametrize("page", [0, 16])
def test_heads(dtype, hq, hkv, d, page):
    Problem(dtype, hq, hkv, d, [5, 1, 40], [70, 33, 130], page=page, seed=d).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("queries,kv", [([1], [1]), ([1, 1, 1], [0, 1, 2]), ([0, 3, 0], [5, 0, 17]), ([33], [31]), ([64], [64]), ([65], [129]),
                                        ([1] * 9, [0, 15, 16, 17, 31, 32, 33, 63, 65]), ([7, 200, 1], [300, 200, 1]), ([130], [513])])
def test_lengths(dtype, page, causal, queries, kv):
    Problem(dtype, 4, 2, 64, queries, kv, page=page, causal=causal, seed=len(kv), elsewhere=3.0).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_and_their_last_tokens(dtype):
    Problem(dtype, 8, 2, 128, [260, 5, 77], [260, 5, 77], causal=True).check()
    Problem(dtype, 8, 2, 128, [16, 3, 50], [400, 140, 60], page=16, causal=True).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv", [(17, 1), (33, 1), (48, 1), (64, 2), (64, 1), (7, 1)])
def test_large_and_odd_groups(dtype, hq, hkv):
    """Groups that fill, split and overlap blocks of 16 and 32 rows, with one query and a few."""
    Problem(dtype, hq, hkv, 64, [1] * 5, [0, 40, 17, 129, 300], page=16, elsewhere=3.0).check()
    Problem(dtype, hq, hkv, 64, [3, 11], [150, 30], causal=True, seed=1).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("g", [1, 3, 4])
def test_parts_of_the_rows(dtype, g):
    """Long prompts, whose rows are cut into parts, some of them empty, causal and not, beside one without queries."""
    Problem(dtype, 2 * g, 2, 64, [1100 // g, 0, 3, 260], [1100 // g, 50, 300, 260], causal=True, seed=g).check()
    Problem(dtype, g, 1, 64, [900 // g], [20], seed=g).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_windows_of_many_sequences(dtype, d, causal):
    """Some dozens of rows over many sequences, with and without pages: none, one and several tiles of tokens, rows that end in a block."""
    queries = [(7 * i) % 41 for i in range(18)]
    kv = [max((97 * i) % 700, 0) for i in range(18)]
    Problem(dtype, 6, 2, d, queries, kv, page=16 if causal else 0, causal=causal, seed=d, elsewhere=0.0 if causal else 2.0).check()


def test_one_window_over_a_long_cache():
    """More tokens than a workgroup's wavefronts take at once, and shared samples over them."""
    Problem("bf16", 4, 1, 64, [60], [9000], page=16, causal=True).check()
    Problem("bf16", 4, 4, 128, [40, 33], [5000, 3100]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_last_queries_of_the_last_row(dtype):
    """The queries end where their tensor does, in the middle of a block."""
    for n in (9, 17, 40):
        Problem(dtype, 4, 1, 128, [n], [64]).check()
        Problem(dtype, 12, 1, 128, [n], [64], causal=True).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_queries_than_tokens(dtype):
    """Causal queries ahead of the first token see nothing; their lse is -inf."""
    Problem(dtype, 4, 2, 64, [40, 9], [25, 3], causal=True).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay,old", [(1.0, True), (0.0, True), (0.5, True), (-1.0, True), (1.0, False), (0.25, False)])
def test_decay(dtype, decay, old):
    p = Problem(dtype, 4, 1, 64, [3, 8], [100, 37], decay=decay, old=old, stride_pad=9)
    if decay < 0:  # a difference of two sums: bounded by their sum
        ref, size = p.reference()
        got = p.launch(p.up()).double().cpu()
        bound = 3e-5 * (size / 60).clamp(min=1.0)[:, None, None] * (ref + 2 * p.old.double())
        for b, n in enumerate(p.kv):
            assert bool(((got[b, :, :n] - ref[b, :, :n]).abs() <= bound[b, :, :n]).all())
        return
    if decay == 0:
        p.old.fill_(float("nan"))  # not read
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_bounds_and_strides(dtype):
    p = Problem(dtype, 8, 2, 72, [4, 1], [90, 20], lead=3, spare=2, stride_pad=5, strides=True)
    s = p.up()
    want = p.launch(s).clone()
    p.check(want)
    s["out"].copy_(s["old"])
    s["old"] = s["out"]
    got = p.launch(s)
    for b, n in enumerate(p.kv):
        assert torch.equal(got[b, :, :n], want[b, :, :n])
        assert torch.equal(got[b, :, n:].cpu(), p.old[b, :, n:])
    s = p.up()
    assert Problem.check(p, p.launch(s, max_query=57, max_kv=95)) is None  # larger bounds than the lengths


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_queries_that_see_nothing(dtype):
    p = Problem(dtype, 4, 2, 64, [6], [50])
    p.lse[2] = -math.inf
    p.lse[4, 1] = -math.inf
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_a_query_does_not_see(dtype):
    """A causal query that is NaN or infinite touches only the tokens that it sees."""
    p = Problem(dtype, 4, 2, 64, [70], [150], causal=True)
    clean = p.launch(p.up()).cpu()
    for bad in (float("nan"), float("inf")):
        s = p.up()
        s["q"][10] = bad
        got = p.launch(s).cpu()
        assert torch.isfinite(got[:, :, 91:150]).all()
        assert torch.allclose(got[:, :, 91:150], clean[:, :, 91:150], rtol=1e-6, atol=0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.5, 0.01])
def test_scale_and_large_scores(dtype, scale):
    Problem(dtype, 4, 1, 128, [5], [200], scale=scale, peak=1.5).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_queries_over_few_tokens(dtype):
    Problem(dtype, 4, 1, 64, [700], [40]).check()
    Problem(dtype, 8, 1, 64, [300, 2], [3, 500], causal=True).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences(dtype):
    kv = [(37 * i) % 90 for i in range(150)]
    Problem(dtype, 4, 2, 64, [1] * 150, kv, page=16, elsewhere=4.0).check()
    Problem(dtype, 4, 2, 64, [i % 3 for i in range(150)], kv, elsewhere=4.0).check()


def test_shared_pages():
    """Sequences that share a page have weights of their own."""
    p = Problem("bf16", 4, 2, 64, [2, 3], [40, 40], page=16)
    p.pages[3:6] = p.pages[0:3]
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_to_the_bit_and_replays(dtype):
    from paper_2502_02534_amd import binding as B
    p = Problem(dtype, 8, 2, 64, [90, 3], [120, 300], old=True)
    s = p.up()
    want = p.launch(s).clone()
    p.check(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = p.launch(s, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    ws = torch.empty(max(256, B.accumulate_kv_weights_workspace_size(p.desc, p.total, p.max_query, p.max_kv)), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        p.launch(s, ws=ws)
    q = s["q"].clone()
    for n in range(4):
        s["q"].copy_(q * (1.0 if n % 2 == 0 else 0.5))
        s["out"].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        again = s["out"].clone()
        p.launch(s)
        torch.cuda.synchronize()
        for b, m in enumerate(p.kv):
            assert torch.equal(again[b, :, :m], s["out"][b, :, :m]), n
            if n % 2 == 0:
                assert torch.equal(again[b, :, :m], want[b, :, :m])


def test_far_keys():
    """Keys past 2^31 elements, contiguous and paged."""
    from paper_2502_02534_amd import binding as B
    hkv, d, n = 2, 64, 40
    far = (2 ** 31 // (hkv * d)) // PAGE * PAGE + 160
    pool = torch.zeros((far + 64) * hkv * d, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(0)
    q = torch.randn((2, 4, d), generator=g, device=DEV).to(torch.bfloat16)
    lse = torch.full((2, 4), 5.0, device=DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    keys = torch.randn((n, hkv, d), generator=g, device=DEV).to(torch.bfloat16)
    want = torch.exp(torch.einsum("ijgd,tjd->ijgt", q.double().unflatten(1, (2, 2)), keys.double()) / 8 - 5.0).sum((0, 2))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    for page in (0, 16):
        if page:
            paged = pool.view(-1, hkv, PAGE, d)
            table = i32([far // PAGE + x for x in (2, 0, 1)])
            for t in range(n):
                paged[int(table[t // PAGE]), :, t % PAGE] = keys[t]
            starts = i32([0, 3])
        else:
            pool.view(-1, hkv, d)[far:far + n] = keys
            table, starts = None, i32([far, far + n])
        out = torch.zeros((1, hkv, n), device=DEV)
        desc = B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=4, num_kv_heads=hkv, head_dim=d, num_prompts=1, page_size=page, causal=False)
        B.accumulate_kv_weights(desc, q, pool, i32([0, 2]), i32([n]), starts, table, lse, 2, 2, n, 0.0, None, out, n, ws)
        assert bool(((out[0].double() - want).abs() <= 3e-5 * want).all()), page


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries,kv,causal", [([700, 3, 1, 0], [700, 3, 1, 2], True), ([2, 400, 30], [900, 400, 31], True), ([300, 1], [40, 1500], False)])
@pytest.mark.parametrize("spare", [0, 2000])
def test_one_long_sequence_among_short_ones(dtype, queries, kv, causal, spare):
    """The parts are made for the queries that there are, or (`spare`: total_queries is more than the sequences have) for each
    sequence's most: the short ones' parts are empty, or one row block's share."""
    from paper_2502_02534_amd import binding as B
    p = Problem(dtype, 4, 2, 64, queries, kv, causal=causal, spare=spare, seed=91)
    assert B.accumulate_kv_weights_workspace_size(p.desc, p.total, p.max_query, p.max_kv) > 256  # (parts)
    p.check()
