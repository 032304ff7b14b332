"""`build_page_tables` and `write_prompt_kv` through the C ABI against loops over requests on the host (whole
numbers and copies: every entry has to be equal)."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def host_tables(lens, held_lens, held, free, begin, page):
    """held[i]: the pages of request i."""
    taken, short, needed = begin, False, 0
    tables, out, slots = [], [], []
    for want, had, mine in zip(lens, held_lens, held):
        want = max(want, had, 0)
        need = max(0, -(-want // page) - len(mine))
        needed += need
        short = short or needed > len(free) - begin
        if need and short:
            tables.append(list(mine))
            out.append(had)
            continue
        tables.append(list(mine) + free[taken:taken + need])
        taken += need
        out.append(want)
        slots.extend(tables[-1][t // page] * page + t % page for t in range(had, want))
    return tables, out, slots, taken


def check(lens, past=None, free_count=None, begin=0, page=16, seed=0, spare=5, slack=True, null_slots=False, stream=None):
    from paper_2502_02534_amd import binding as B
    rng = random.Random(seed)
    n = len(lens)
    had = past or [0] * n
    held_counts = [-(-x // page) + (rng.randrange(2) if slack and past else 0) for x in had]  # a page ahead now and then
    need = sum(max(0, -(-max(a, b, 0) // page) - h) for a, b, h in zip(lens, had, held_counts))
    count = begin + (need if free_count is None else free_count)
    ids = list(range(sum(held_counts) + count))
    rng.shuffle(ids)
    first = _starts(held_counts)
    held = [ids[first[i]:first[i + 1]] for i in range(n)]
    free = ids[first[-1]:]
    tables, want_lens, want_slots, taken = host_tables(lens, had, held, free, begin, page)
    print(f"tables n {n} page {page} need {need} free {len(free)} begin {begin} tokens {len(want_slots)}", flush=True)
    max_pages, max_tokens = sum(map(len, tables)) + spare, len(want_slots) + spare
    page_indptr, lens_out, new_indptr = (torch.full((k,), -9, dtype=torch.int32, device=DEV) for k in (n + 1, n, n + 1))
    pages = torch.full((max_pages,), -9, dtype=torch.int32, device=DEV)
    slots = torch.full((max_tokens,), -9, dtype=torch.int64, device=DEV)
    end = _i32([-9])
    ws = torch.empty(B.build_page_tables_workspace_size(n), dtype=torch.uint8, device=DEV)
    held_args = (_i32(had), _i32(first), _i32(ids[:first[-1]] or [0])) if past else (None, None, None)
    begin_arg = _i32([begin]) if begin else None
    free_arg = _i32(free or [0])
    torch.cuda.synchronize()
    B.build_page_tables(n, page, _i32(lens), *held_args, free_arg, len(free), begin_arg, max_pages, max_tokens, page_indptr,
                        pages, lens_out, new_indptr, None if null_slots else slots, end, ws, stream)
    torch.cuda.synchronize()
    assert page_indptr.tolist() == _starts([len(t) for t in tables])
    assert pages.tolist() == [x for t in tables for x in t] + [-1] * spare
    assert lens_out.tolist() == want_lens
    assert new_indptr.tolist() == _starts([a - b for a, b in zip(want_lens, had)])
    assert slots.tolist() == ([-9] * max_tokens if null_slots else want_slots + [-1] * spare)
    assert end.tolist() == [taken]


@pytest.mark.parametrize("n", [1, 2, 8, 63, 64, 65, 1023, 1024, 1025, 2500, 5000])
def test_requests_from_nothing(n):
    rng = random.Random(n)
    check([rng.randrange(0, 70) for _ in range(n)], seed=n)


@pytest.mark.parametrize("n", [1, 7, 130, 1024, 2049])
def test_requests_that_grow(n):
    rng = random.Random(n)
    past = [rng.randrange(0, 90) for _ in range(n)]
    check([x + rng.randrange(0, 30) for x in past], past, seed=n)
    check([x + 1 for x in past], past, seed=n + 1, slack=False)


@pytest.mark.parametrize("page", [1, 7, 16, 64, 65536])
def test_page_sizes(page):
    check([0, 1, page, page + 1, 3 * page + 2] if page < 1000 else [0, 1, 70000], page=page)
    check([5, 40, 41], [5, 20, 40], page=page, seed=3)


@pytest.mark.parametrize("n", [9, 1500])
@pytest.mark.parametrize("share", [0.0, 0.3, 0.999])
def test_a_free_list_that_runs_out(n, share):
    rng = random.Random(n)
    past = [rng.randrange(0, 50) for _ in range(n)]
    lens = [x + rng.choice([0, 1, 40]) for x in past]
    need = sum(max(0, -(-a // 16) - -(-b // 16)) for a, b in zip(lens, past))
    check(lens, past, free_count=int(need * share), slack=False, seed=n)
    check(lens, past, free_count=int(need * share), begin=13, slack=False, seed=n + 1)


def test_odd_lengths():
    check([0, 0, 0])                                     # nothing to hold
    check([-5, 3, -(1 << 31), 17])                       # negative lengths count as 0
    check([3, 100], [50, 20], seed=4)                    # shorter than what is held: nothing is given up
    check([100000, 1, 65, 0, 40000], spare=0)            # long ones, arrays of exactly the size
    check([(1 << 31) - 1, 5, (1 << 31) - 1, 16], free_count=10)  # asks for more than there is, several times over
    check([64, 5], null_slots=True)


def test_a_chain_of_calls_deals_from_one_list():
    """free_end of the prompts' tables is free_begin of the samples'."""
    from paper_2502_02534_amd import binding as B
    free = _i32(list(range(100, 200)))
    ends = [torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2)]
    pages = []
    for call, lens in enumerate(([40, 17], [1, 16, 33])):
        n = len(lens)
        ip, idx, lo, ni = _i32([0] * (n + 1)), _i32([0] * 8), _i32([0] * n), _i32([0] * (n + 1))
        ws = torch.empty(B.build_page_tables_workspace_size(n), dtype=torch.uint8, device=DEV)
        B.build_page_tables(n, 16, _i32(lens), None, None, None, free, 100, ends[0] if call else None, 8, 0, ip, idx, lo, ni, None,
                            ends[call], ws)
        pages.append(idx)
    torch.cuda.synchronize()
    assert pages[0].tolist() == [100, 101, 102, 103, 104, -1, -1, -1]
    assert pages[1].tolist() == [105, 106, 107, 108, 109, -1, -1, -1]
    assert ends[1].tolist() == [10]


def test_arrays_that_are_too_short_are_not_overrun():
    from paper_2502_02534_amd import binding as B
    pages, slots = _i32([-9] * 10), torch.full((40,), -9, dtype=torch.int64, device=DEV)
    ip, lo, ni, end = _i32([0, 0, 0]), _i32([0, 0]), _i32([0, 0, 0]), _i32([0])
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    B.build_page_tables(2, 16, _i32([64, 64]), None, None, None, _i32(list(range(20))), 20, None, 6, 30, ip, pages, lo, ni, slots,
                        end, ws)
    torch.cuda.synchronize()
    assert pages.tolist() == [0, 1, 2, 3, 4, 5] + [-9] * 4 and ip.tolist() == [0, 4, 8]
    assert slots.tolist() == list(range(30)) + [-9] * 10


def test_tables_on_another_stream_and_in_a_graph():
    from paper_2502_02534_amd import binding as B
    check([30, 50, 1], [16, 0, 1], stream=torch.cuda.Stream())
    lens, free = _i32([30, 50]), _i32(list(range(8)))
    ip, idx, lo, ni, end = _i32([0] * 3), _i32([0] * 6), _i32([0] * 2), _i32([0] * 3), _i32([0])
    slots = torch.zeros(80, dtype=torch.int64, device=DEV)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    call = lambda: B.build_page_tables(2, 16, lens, None, None, None, free, 8, None, 6, 80, ip, idx, lo, ni, slots, end, ws)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for a, b in ((30, 50), (1, 2), (64, 16)):
        lens.copy_(_i32([a, b]))
        graph.replay()
        torch.cuda.synchronize()
        want = [t for t in range(a)] + [16 * -(-a // 16) + t for t in range(b)]
        assert slots.tolist() == want + [-1] * (80 - a - b)
        torch.randn(100, device=DEV).sum().item()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,d", [(1, 8), (1, 64), (2, 40), (8, 128), (3, 256), (5, 80)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("fused", [False, True])
def test_write_prompt_kv(dtype, hkv, d, page, fused):
    from paper_2502_02534_amd import binding as B
    g = torch.Generator().manual_seed(hkv + d)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    for tokens in (1, 2, 17, 301):
        num_pages = (tokens // 16 + 4) if page else tokens + 9
        slots = torch.randperm(num_pages * (page or 1), generator=g)[:tokens]
        slots[::5] = -1                                         # padding is skipped
        if tokens > 2:
            slots[1] = num_pages * (page or 1) + 3                # and so is what lies outside the pool
        wide = torch.randn((tokens, 2 * hkv * d + 16), generator=g).to(t)
        k, v = wide[:, :hkv * d].unflatten(1, (hkv, d)), wide[:, hkv * d:2 * hkv * d].unflatten(1, (hkv, d))
        shape = (num_pages, hkv, 16, d) if page else (num_pages, hkv, d)
        pools = [torch.full(shape, 7.0, dtype=t) for _ in range(2)]
        dev_pools = [x.to(DEV) for x in pools]
        for x, pool in ((k, pools[0]), (v, pools[1])):
            for i, s in enumerate(slots.tolist()):
                if 0 <= s < num_pages * (page or 1):
                    if page:
                        pool[s // 16, :, s % 16] = x[i]
                    else:
                        pool[s] = x[i]
        desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=hkv, num_kv_heads=hkv, head_dim=d,
                                  num_prompts=1, page_size=page, kv_stride=wide.stride(0) if fused else 0)
        wd = wide.to(DEV)
        kd, vd = wd[:, :hkv * d], wd[:, hkv * d:2 * hkv * d]
        if not fused:
            kd, vd = kd.contiguous(), vd.contiguous()
        B.write_prompt_kv(desc, kd, vd, slots.to(DEV), tokens, num_pages, *dev_pools)
        torch.cuda.synchronize()
        for a, b in zip(dev_pools, pools):
            assert torch.equal(a.cpu(), b), (tokens, page)


def test_write_past_two_gigabytes():
    from paper_2502_02534_amd import binding as B
    hkv, d = 8, 128
    pages = (1 << 31) // (hkv * 16 * d) + 40
    pool = torch.zeros((pages, hkv, 16, d), dtype=torch.bfloat16, device=DEV)
    other = torch.zeros((64, hkv, 16, d), dtype=torch.bfloat16, device=DEV)
    k = torch.randn((20, hkv, d), device=DEV, dtype=torch.bfloat16)
    slots = torch.arange(pages * 16 - 20, pages * 16, device=DEV)
    desc = B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=hkv, num_kv_heads=hkv, head_dim=d, num_prompts=1, page_size=16)
    B.write_prompt_kv(desc, k, k, slots, 20, pages, pool, pool)
    torch.cuda.synchronize()
    assert torch.equal(pool[slots // 16, :, slots % 16], k)
    assert int((pool[: pages - 2] != 0).any()) == 0
    del other
