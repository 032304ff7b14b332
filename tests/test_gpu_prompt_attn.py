"""`prompt_attn` through the C ABI against softmax(q K^T * scale) V in 64 bits, row by row.

Tolerances, with A = sum_t p_t |v_t| of a row and channel (>= |ref|) and M = the largest scale * sum_c |q_c k_c| of
the tokens that the row sees:
  e     the relative error of a probability in fp32 is the absolute error of its score, which the summation over
        the channels makes a few units of 2^-24 M; e = 1e-5 max(1, M / 60) allows three of them (and more below 60)
  bf16  err <= (2 * 2^-8 + 20 e) A + 1e-6: the result is rounded to 8 significant bits once (2^-8 relative), and so are
        the probabilities on their way into the second product (2^-8 of each term); 1e-6 for results near zero
  fp32  err <= e A + 1e-6, the library's rule for fp32 with the terms' magnitude in place of the result's
  lse   err <= 1e-4 max(1, M / 60), -inf where nothing is seen."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PAGE = 16


class Problem:
    """new[b] new tokens after past[b] cached ones (past may be negative: more queries than KV tokens)."""

    def __init__(self, dtype, hq, hkv, d, new, past, page=0, causal=True, fused=False, seed=0, scale=0.0, spare=0, peak=1.0):
        from paper_2502_02534_amd import binding as B
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.hq, self.hkv, self.d, self.new, self.page, self.causal = dtype, hq, hkv, d, new, page, causal
        self.kv = [a + b for a, b in zip(new, past)]
        assert min(self.kv) >= 0
        t = torch.float32 if dtype == "f32" else torch.bfloat16
        draw = lambda *shape: torch.randn(shape, generator=g).to(t)  # noqa: E731
        self.total = sum(new)
        ptr = lambda lens: torch.tensor([0] + lens).cumsum(0).to(torch.int32)  # noqa: E731
        self.query_indptr, self.kv_lens = ptr(new), torch.tensor(self.kv, dtype=torch.int32)
        self.q_stride = self.kv_stride = 0
        rows = max(self.total, 1)
        if fused:
            assert not page and not any(past)
            wide = draw(rows, (hq + 2 * hkv) * d + 8)
            self.q = wide[:, : hq * d].unflatten(1, (hq, d))
            self.k = wide[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
            self.v = wide[:, (hq + hkv) * d:(hq + 2 * hkv) * d].unflatten(1, (hkv, d))
            self.wide = wide
            self.q_stride = self.kv_stride = wide.stride(0)
            self.kv_indptr, self.pages = self.query_indptr, None
        elif page:
            self.q = draw(rows, hq, d)
            held = [-(-n // PAGE) for n in self.kv]
            pool = sum(held) + 3
            self.kv_indptr = ptr(held)
            self.pages = torch.randperm(pool, generator=g)[: max(sum(held), 1)].to(torch.int32)
            self.k, self.v = draw(pool, hkv, PAGE, d), draw(pool, hkv, PAGE, d)
            # what lies past a prompt's end in its last page, or in no prompt's page, is never read
            live = torch.zeros(pool, PAGE, dtype=torch.bool)
            for b, n in enumerate(self.kv):
                for t0 in range(n):
                    live[self.pages[self.kv_indptr[b] + t0 // PAGE], t0 % PAGE] = True
            self.k[~live[:, None, :, None].expand_as(self.k)] = float("nan")
            self.v[~live[:, None, :, None].expand_as(self.v)] = float("inf")
        else:
            self.q = draw(rows, hq, d)
            self.kv_indptr, self.pages = ptr(self.kv), None
            self.k, self.v = draw(max(sum(self.kv), 1), hkv, d), draw(max(sum(self.kv), 1), hkv, d)
        if peak != 1.0:
            self.q.mul_(peak)
        self.scale = scale if scale > 0 else 1.0 / math.sqrt(d)
        self.spare = spare
        self.desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=hq, num_kv_heads=hkv,
                                       head_dim=d, num_prompts=len(new), page_size=page, causal=causal, sm_scale=scale,
                                       q_stride=self.q_stride, kv_stride=self.kv_stride)

    def rows_of(self, b, which):
        """K or V of prompt b, [kv_len, hkv, d]."""
        x, n, at = (self.k if which == "k" else self.v), self.kv[b], int(self.kv_indptr[b])
        if self.page:
            ids = self.pages[at:at + -(-n // PAGE)].long()
            return x[ids].transpose(1, 2).reshape(-1, self.hkv, self.d)[:n]
        return x[at:at + n]

    def reference(self):
        out = torch.zeros(self.total, self.hq, self.d, dtype=torch.float64)
        mass = torch.zeros_like(out)
        lse = torch.full((self.total, self.hq), -math.inf, dtype=torch.float64)
        self.size = torch.zeros(self.total, self.hq, dtype=torch.float64)
        g = self.hq // self.hkv
        for b, n in enumerate(self.new):
            k, v = self.rows_of(b, "k").double(), self.rows_of(b, "v").double()
            for i in range(n):
                r = int(self.query_indptr[b]) + i
                see = max(0, min(self.kv[b], self.kv[b] - n + i + 1)) if self.causal else self.kv[b]
                if see == 0:
                    continue
                for j in range(self.hkv):
                    q = self.q[r, j * g:(j + 1) * g].double()
                    s = q @ k[:see, j].T * self.scale
                    self.size[r, j * g:(j + 1) * g] = (q.abs() @ k[:see, j].abs().T * self.scale).amax(1)
                    total = torch.logsumexp(s, 1)
                    p = torch.exp(s - total[:, None])
                    lse[r, j * g:(j + 1) * g] = total
                    out[r, j * g:(j + 1) * g] = p @ v[:see, j]
                    mass[r, j * g:(j + 1) * g] = p @ v[:see, j].abs()
        return out, mass, lse

    def tolerance(self, mass):
        e = 1e-5 * (self.size / 60).clamp(min=1.0)[:, :, None]
        return ((2 * 2.0 ** -8 + 20 * e) if self.dtype == "bf16" else e) * mass + 1e-6

    def lse_tolerance(self):
        return 1e-4 * (self.size / 60).clamp(min=1.0)

    def run(self, with_lse=True, max_query=None, max_kv=None, stream=None):
        from paper_2502_02534_amd import binding as B
        up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
        if self.q_stride:
            wide = self.wide.to(DEV)
            hq, hkv, d = self.hq, self.hkv, self.d
            q = wide[:, : hq * d].unflatten(1, (hq, d))
            k = wide[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
            v = wide[:, (hq + hkv) * d:(hq + 2 * hkv) * d].unflatten(1, (hkv, d))
        else:
            q, k, v = up(self.q), up(self.k), up(self.v)
        mq, mk = max_query or max(self.new), max_kv or max(self.kv)
        rows = self.total + self.spare
        size = B.prompt_attn_workspace_size(self.desc, rows, mq, mk)
        assert size > 0
        ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)  # NaN as fp32
        out = torch.full((max(rows, 1), self.hq, self.d), 7.0, dtype=q.dtype, device=DEV)
        lse = torch.full((max(rows, 1), self.hq), 7.0, device=DEV) if with_lse else None
        args = [up(self.query_indptr), up(self.kv_lens), up(self.kv_indptr), up(self.pages)]
        torch.cuda.synchronize()
        B.prompt_attn(self.desc, q, k, v, *args, rows, mq, mk, out, lse, ws, stream)
        torch.cuda.synchronize()
        return out.cpu(), None if lse is None else lse.cpu()

    def check(self, **kw):
        print(f"prompt {self.dtype} {self.hq}/{self.hkv}/{self.d} new {self.new[:6]} kv {self.kv[:6]} page {self.page} "
              f"causal {self.causal}", flush=True)
        out, lse = self.run(**kw)
        ref, mass, ref_lse = self.reference()
        assert bool((out[self.total:] == 7.0).all())  # nothing past the last query is written, bar the empty call's
        err, got = (out[: self.total].double() - ref).abs(), out[: self.total]
        assert bool(torch.isfinite(got.float()).all())
        tol = self.tolerance(mass)
        worst = float((err - tol).max()) if err.numel() else 0.0
        assert worst <= 0, (worst, float(err.max()))
        if lse is not None:
            none = torch.isinf(ref_lse)
            assert torch.equal(torch.isneginf(lse[: self.total]), none)
            assert bool(((lse[: self.total].double() - ref_lse).abs() <= self.lse_tolerance())[~none].all())
            assert bool((got[none] == 0).all())
            assert bool((lse[self.total:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (8, 8, 128), (6, 2, 128), (32, 8, 64), (5, 1, 8), (2, 2, 40), (4, 4, 72),
                                      (4, 2, 96), (2, 1, 136), (3, 1, 256), (40, 2, 128)])
def test_heads_and_dimensions(dtype, hq, hkv, d):
    Problem(dtype, hq, hkv, d, [37, 1, 70], [0, 0, 0], seed=hq + d).check()
    Problem(dtype, hq, hkv, d, [5, 33], [40, 7], page=PAGE, seed=hq + d + 1).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_lengths_at_the_edges_of_tiles(dtype, d, n):
    Problem(dtype, 4, 2, d, [n], [0], seed=n).check()
    Problem(dtype, 2, 1, d, [n, 3], [17, 64], page=PAGE, seed=n + 1).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, PAGE])
def test_empty_prompts_and_rows_that_see_nothing(dtype, page):
    Problem(dtype, 4, 2, 128, [0, 9, 0, 0, 40, 0], [0, 0, 3, 0, -25, 0], page=page, seed=5).check()
    Problem(dtype, 4, 2, 64, [6, 3], [-6, 10], page=page, seed=6).check()      # one prompt has no KV at all
    Problem(dtype, 4, 2, 64, [6, 3], [-6, 10], page=page, causal=False, seed=6).check()
    Problem(dtype, 4, 2, 128, [0, 0], [5, 0], page=page, spare=3, seed=7).check()  # no query at all


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, PAGE])
@pytest.mark.parametrize("d", [64, 128, 80])
def test_without_a_causal_mask(dtype, page, d):
    Problem(dtype, 6, 3, d, [50, 7, 129], [0, 100, 31], page=page, causal=False, seed=d).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 48])
def test_slices_of_one_projection(dtype, d):
    Problem(dtype, 8, 2, d, [100, 1, 61], [0, 0, 0], fused=True, seed=d, spare=2).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, PAGE])
def test_few_new_tokens_over_a_long_cache(dtype, d, page):
    # one token each, and a handful: the tokens are cut into splits that are joined afterwards
    Problem(dtype, 8, 2, d, [1, 1, 1], [1500, 3, 700], page=page, seed=1).check()
    Problem(dtype, 4, 1, d, [7, 1, 0, 12], [2100, 0, 50, 333], page=page, seed=2, peak=4.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_longer_prompt(dtype):
    Problem(dtype, 4, 2, 128, [700, 1, 333], [0, 200, 0], seed=3, peak=3.0).check()
    Problem(dtype, 8, 1, 64, [450], [1111], page=PAGE, seed=4, peak=3.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_short_prompts(dtype):
    new = [(7 * i) % 23 for i in range(150)]
    past = [(5 * i) % 41 for i in range(150)]
    Problem(dtype, 4, 2, 64, new, past, page=PAGE, seed=8).check()
    Problem(dtype, 2, 1, 128, new, past, seed=9).check()


def test_scale_bounds_and_no_log_sum_exp():
    Problem("bf16", 4, 2, 128, [65], [10], seed=11, scale=0.03).check(with_lse=False)
    Problem("f32", 4, 2, 64, [65, 3], [10, 0], seed=12, scale=0.3).check(max_query=500, max_kv=4000)
    Problem("bf16", 4, 2, 64, [65, 3], [10, 0], seed=12).check(max_query=500, max_kv=4000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 40])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_a_row_does_not_see_does_not_matter(dtype, d, bad):
    """Rows before a token whose K and V are not finite get what they get without it."""
    for n, x in ((60, 41), (200, 150), (33, 0)):
        p = Problem(dtype, 4, 2, d, [n], [0], seed=n)
        p.k[x:], p.v[x:] = bad, bad
        print(f"unseen {dtype} {d} {n} from {x}: {bad}", flush=True)
        out, lse = p.run()
        p.new, p.kv = [x], [x]  # the reference of the rows that see none of it
        p.total = x
        ref, mass, ref_lse = p.reference()
        assert bool(((out[:x].double() - ref).abs() <= p.tolerance(mass)).all())
        assert bool(((lse[:x].double() - ref_lse).abs() <= p.lse_tolerance()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype, d):
    n = 100
    p = Problem(dtype, 4, 2, d, [n], [0], seed=d)
    p.v[50, 0, 3] = float("inf")
    p.v[70, 1, 5] = float("-inf")
    p.v[80, 0, 7] = float("nan")
    out, _ = p.run()
    out = out.float()
    for h in range(4):
        j = h // 2
        want = torch.zeros(n, d)
        if j == 0:
            want[50:, 3], want[80:, 7] = math.inf, math.nan
        else:
            want[70:, 5] = -math.inf
        odd = want != 0
        assert torch.equal(torch.isnan(out[:, h]), torch.isnan(want))
        assert bool(torch.isfinite(out[:, h][~odd]).all())
        assert torch.equal(out[:, h][odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_score_peaks_and_large_values(dtype):
    # one token far ahead of the rest in some rows, values up to 2^100
    p = Problem(dtype, 4, 2, 128, [150], [30], seed=21, peak=12.0)
    p.k[3] *= 4.0
    p.check()
    p = Problem(dtype, 4, 2, 64, [9], [1300], seed=22)
    p.v.mul_(2.0 ** 100)
    out, _ = p.run()
    ref, mass, _ = p.reference()
    assert bool(((out.double() - ref).abs() <= p.tolerance(mass)).all())


def test_shared_pages_and_determinism():
    """Two prompts whose tables begin with the same pages (a shared context), and the same bits on every call."""
    for dtype in ("bf16", "f32"):
        p = Problem(dtype, 8, 2, 128, [20, 30], [64, 64], page=PAGE, seed=31)
        shared = p.pages.clone()
        shared[int(p.kv_indptr[1]):int(p.kv_indptr[1]) + 4] = shared[:4]
        p.pages = shared
        p.check()
        a, b = p.run(), p.run()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_another_stream_and_a_captured_graph():
    from paper_2502_02534_amd import binding as B
    p = Problem("bf16", 8, 2, 128, [3, 40], [900, 10], page=PAGE, seed=41)
    want, want_lse = p.run()
    side = torch.cuda.Stream()
    got, got_lse = p.run(stream=side)
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse)
    q, k, v = p.q.to(DEV), p.k.to(DEV), p.v.to(DEV)
    ints = [x.to(DEV) for x in (p.query_indptr, p.kv_lens, p.kv_indptr, p.pages)]
    out, lse = torch.zeros_like(q), torch.zeros(p.total, p.hq, device=DEV)
    ws = torch.empty(B.prompt_attn_workspace_size(p.desc, p.total, 40, 910), dtype=torch.uint8, device=DEV)
    call = lambda: B.prompt_attn(p.desc, q, k, v, *ints, p.total, 40, 910, out, lse, ws)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want) and torch.equal(lse.cpu(), want_lse)
        torch.randn(1000, device=DEV).sum().item()


def test_kv_past_two_gigabytes():
    """Element offsets beyond 2^31 in a contiguous cache: the last prompt's tokens are read from their own place."""
    from paper_2502_02534_amd import binding as B
    hkv, d, far = 8, 128, (1 << 31) // (8 * 128) + 100
    k = torch.zeros((far + 64, hkv, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    g = torch.Generator(device=DEV).manual_seed(1)
    k[far:] = torch.randn((64, hkv, d), generator=g, device=DEV, dtype=torch.bfloat16)
    v[far:] = torch.randn((64, hkv, d), generator=g, device=DEV, dtype=torch.bfloat16)
    q = torch.randn((64, hkv, d), generator=g, device=DEV, dtype=torch.bfloat16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    desc = B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=hkv, num_kv_heads=hkv, head_dim=d, num_prompts=1)
    ws = torch.empty(B.prompt_attn_workspace_size(desc, 64, 64, 64), dtype=torch.uint8, device=DEV)
    far_out, near_out = torch.empty_like(q), torch.empty_like(q)
    B.prompt_attn(desc, q, k, v, i32(0, 64), i32(64), i32(far, far + 64), None, 64, 64, 64, far_out, None, ws)
    B.prompt_attn(desc, q, k[far:].clone(), v[far:].clone(), i32(0, 64), i32(64), i32(0, 64), None, 64, 64, 64, near_out, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(far_out, near_out) and float(near_out.float().abs().sum()) > 0
