"""`prompt_attn` where its launch changes form: parts of more than 64 prompts, tiles in pairs, blocks of every width of
head, values that are not finite in a part or among long prompts.  Reference and tolerances are those of
tests/test_gpu_prompt_attn.py, the reference over whole matrices."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_prompt_attn import DEV, PAGE, Problem  # noqa: E402

pytestmark = pytest.mark.gpu


class Whole(Problem):
    def reference(self):
        out = torch.zeros(self.total, self.hq, self.d, dtype=torch.float64)
        mass = torch.zeros_like(out)
        lse = torch.full((self.total, self.hq), -math.inf, dtype=torch.float64)
        self.size = torch.zeros(self.total, self.hq, dtype=torch.float64)
        g = self.hq // self.hkv
        for b, n in enumerate(self.new):
            L, r = self.kv[b], int(self.query_indptr[b])
            if n == 0 or L == 0:
                continue
            k, v = self.rows_of(b, "k").double(), self.rows_of(b, "v").double()
            sees = torch.ones(n, L, dtype=torch.bool)
            if self.causal:
                sees = torch.arange(L)[None, :] <= L - n + torch.arange(n)[:, None]
            for h in range(self.hq):
                j = h // g
                q = self.q[r:r + n, h].double()
                s = (q @ k[:, j].T * self.scale).masked_fill(~sees, -math.inf)
                total = torch.logsumexp(s, 1)
                p = torch.exp(s - total[:, None]).nan_to_num(0.0)  # (rows that see nothing)
                self.size[r:r + n, h] = (q.abs() @ k[:, j].abs().T * self.scale).masked_fill(~sees, 0.0).amax(1)
                lse[r:r + n, h] = total
                out[r:r + n, h] = p @ v[:, j]
                mass[r:r + n, h] = p @ v[:, j].abs()
        return out, mass, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,n", [(32, 32, 64, 1100), (16, 8, 128, 2150), (16, 16, 40, 2300)])
def test_all_tiles_at_once_in_pairs(dtype, hq, hkv, d, n):
    # 257 to 512 units of 128 rows: those of the second half in the opposite order
    units = (n * hq // hkv // 128 + 1) * hkv
    assert 256 < units <= 512
    Whole(dtype, hq, hkv, d, [n], [0], seed=d).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pairs_of_several_prompts(dtype):
    Whole(dtype, 16, 16, 64, [900, 0, 257, 1, 1130], [0, 40, 100, 300, 0], page=PAGE, seed=51).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,past", [([1300, 1217], [0, 0]), ([900, 0, 1100, 1], [0, 0, 200, 5]), ([40, 2500, 130], [0, 0, 7]),
                                      ([1, 1, 1, 2177], [0, 0, 0, 0])])
def test_units_of_a_few_prompts_by_length(dtype, new, past):
    # more units than run at once: tile by tile across the prompts, also where one has no tiles or one alone has many
    Whole(dtype, 32, 32, 64, new, past, seed=sum(new)).check()


def test_units_by_length_of_a_prompt_of_many_tiles():
    """More tiles than lanes: 32 rows of a token, 4 tokens a tile."""
    Whole("bf16", 32, 1, 64, [2100, 4, 300], [0, 60, 0], seed=53, page=PAGE).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_more_prompts_than_lanes(dtype):
    """Some prompts are one part, some several: their length is found from all the lengths, 64 prompts at a time."""
    new = [(3 * i) % 4 for i in range(100)]
    past = [(97 * i) % 700 if i % 7 else 0 for i in range(100)]
    past[13], past[90] = 2500, 1900
    new[13], new[90] = 2, 1
    p = Whole(dtype, 4, 1, 64, new, past, page=PAGE, seed=52)
    p.check(max_query=3)
    a, b = p.run(), p.run(max_kv=4000)  # a wider bound may cut the parts elsewhere, not change what is computed
    ref, mass, _ = p.reference()
    for out, _ in (a, b):
        assert bool(((out.double() - ref).abs() <= p.tolerance(mass)).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [80, 136, 256])
@pytest.mark.parametrize("page", [0, PAGE])
def test_other_dimensions_over_many_tiles(dtype, d, page):
    Whole(dtype, 4, 2, d, [300, 1, 65], [333, 1000, 0], page=page, seed=d).check()
    Whole(dtype, 8, 8, d, [700, 600], [0, 0], page=page, seed=d + 1).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,past", [([400], [0]), ([3, 2], [1500, 900])])
def test_values_that_are_not_finite_in_parts_and_long_prompts(dtype, d, new, past):
    """Channels that no such value is in keep their result, whichever tile, part or edge it lies in; the others get it where a
    row sees it, and only there."""
    p = Whole(dtype, 4, 2, d, new, past, seed=d)
    clean, _ = p.run()
    L = p.kv[0]
    spots = {2: (L - 1, 0, math.inf), 9: (L // 2, 0, -math.inf), 17: (L - 33, 1, math.nan), 33: (0, 1, math.inf), 50: (L - 2, 1, -math.inf)}
    for c, (t, j, x) in spots.items():
        p.v[t, j, c] = x
    out, _ = p.run()
    ref, _, ref_lse = p.reference()
    want = clean.float().clone()
    for c, (t, j, x) in spots.items():
        for i in range(new[0]):
            if L - new[0] + i >= t:
                want[i, 2 * j:2 * j + 2, c] = x
    odd = ~torch.isfinite(want)
    got = out.float()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])
    keep = torch.ones(d, dtype=torch.bool)
    keep[list(spots)] = False
    assert torch.equal(out[:, :, keep], clean[:, :, keep])
    # a spotted channel of a row that does not see the spot
    q = Whole(dtype, 4, 2, d, new, past, seed=d)
    ref, mass, _ = q.reference()
    assert bool(((out.double() - ref).abs() <= q.tolerance(mass))[~odd].all())


def test_sequences_of_calls_share_a_workspace():
    """What an earlier call left in the workspace, larger or with other parts, is no input of the next."""
    from paper_2502_02534_amd import binding as B
    problems = [Whole("bf16", 8, 2, 128, [1, 1, 1, 1], [3000, 10, 0, 777], seed=61),
                Whole("bf16", 8, 2, 128, [4, 1, 1], [500, 2000, 0], seed=62),
                Whole("f32", 4, 1, 64, [5, 100], [900, 0], seed=63)]
    calls, size = [], 0
    for p in problems:
        mq, mk = max(p.new), max(p.kv)
        size = max(size, B.prompt_attn_workspace_size(p.desc, p.total, mq, mk))
        out, lse = torch.empty_like(p.q, device=DEV), torch.empty(p.total, p.hq, device=DEV)
        ins = [x.to(DEV) for x in (p.q, p.k, p.v, p.query_indptr, p.kv_lens, p.kv_indptr)]
        calls.append((p, ins, (p.total, mq, mk), out, lse))
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    for k in range(2):
        for p, ins, dims, out, lse in calls:
            out.fill_(9.0)
            B.prompt_attn(p.desc, *ins, None, *dims, out, lse, ws)
    torch.cuda.synchronize()
    for p, _, _, out, lse in calls:
        want, want_lse = p.run()
        assert torch.equal(out.cpu(), want) and torch.equal(lse.cpu(), want_lse)
