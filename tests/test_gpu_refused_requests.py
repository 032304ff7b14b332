"""Requests to attention where the free list runs out: the new tokens' rows are packed by what was asked for, so a refused
request's rows keep their places, reach nobody's pages, and get zeros; everybody else gets what a batch without it gets."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HQ, HKV, D, PAGE = 8, 2, 64, 16


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("past,new,free_pages,served", [
    # a turn that needs two pages of the one left is refused; the turns behind it fit their last pages
    ([20, 30, 5, 0], [3, 40, 9, 0], 1, [True, False, True, True]),
    # the first and the last but one of a row of requests, and new requests that get nothing
    ([40, 16, 0, 33, 1], [100, 0, 20, 14, 15], 0, [False, True, False, True, True]),
    ([100, 7, 300], [12, 500, 4], 30, [True, False, True]),
    ([16, 16], [1, 1], 1, [True, False]),
    ([3, 3], [1, 70], 3, [True, False]),
    ([8, 20, 8], [8, 12, 3], 0, [True, True, True])])
def test_refused_requests_touch_nobody(dtype, past, new, free_pages, served):
    from paper_2502_02534_amd import device as dev
    g = torch.Generator().manual_seed(sum(past))
    draw = lambda *shape: torch.randn(shape, generator=g).to(dtype)  # noqa: E731
    n = len(past)
    held = [-(-x // PAGE) for x in past]
    pool_pages = sum(held) + 40
    ids = torch.randperm(pool_pages, generator=g).to(torch.int32)
    k_pool, v_pool = draw(pool_pages, HKV, PAGE, D), draw(pool_pages, HKV, PAGE, D)
    before = k_pool.clone(), v_pool.clone()
    # what the requests hold: nothing goes out beyond its pages
    lens_held, page_starts = _i32(past), _starts(held)
    had = dev.PageTables(_i32(page_starts), ids[:max(sum(held), 1)].to(DEV), lens_held, _i32([0] * (n + 1)), None, _i32([0]))
    free = ids[sum(held):sum(held) + free_pages].to(DEV)
    if not free_pages:
        free = ids[:0].to(DEV)
    tokens, most = sum(new), max(a + b for a, b in zip(past, new))
    t = dev.build_tables(_i32([a + b for a, b in zip(past, new)]), free, sum(held) + free_pages + 2, tokens, held=had)
    q, k, v = draw(tokens, HQ, D), draw(tokens, HKV, D), draw(tokens, HKV, D)
    pools = [x.to(DEV) for x in (k_pool, v_pool)]
    run = dev.DevicePrompts(t, q.to(DEV), k.to(DEV), v.to(DEV), *pools, max(new), most)
    run.out.fill_(5.0)
    run.lse.fill_(5.0)
    print(f"refused {past} + {new} with {free_pages} free", flush=True)
    run.run()
    torch.cuda.synchronize()

    # by hand, in 64 bits
    starts, taken = _starts(new), 0
    out, lse = run.out.double().cpu(), run.lse.double().cpu()
    for b in range(n):
        mine = ids[page_starts[b]:page_starts[b + 1]].tolist()
        rows = slice(starts[b], starts[b + 1])
        if not served[b]:
            assert bool((out[rows] == 0).all()) and bool(torch.isneginf(lse[rows]).all())
            continue
        need = max(0, -(-(past[b] + new[b]) // PAGE) - len(mine))
        mine += free.tolist()[taken:taken + need]
        taken += need
        for i in range(new[b]):
            pos = past[b] + i
            before[0][mine[pos // PAGE], :, pos % PAGE] = k[starts[b] + i]
            before[1][mine[pos // PAGE], :, pos % PAGE] = v[starts[b] + i]
        kk, vv = (x[mine].transpose(1, 2).reshape(-1, HKV, D)[:past[b] + new[b]].double() for x in before)
        for i in range(new[b]):
            see = past[b] + i + 1
            for h in range(HQ):
                s = kk[:see, h // (HQ // HKV)] @ q[starts[b] + i, h].double() / D ** 0.5
                p = torch.softmax(s, 0)
                x = vv[:see, h // (HQ // HKV)]
                # bf16: result and probabilities rounded to 8 bits; scores in fp32
                tol = (2 * 2.0 ** -8 + 2e-4 if dtype == torch.bfloat16 else 1e-5) * (p @ x.abs()) + 1e-6
                assert bool(((out[starts[b] + i, h] - p @ x).abs() <= tol).all()), (b, i, h)
                assert abs(float(lse[starts[b] + i, h] - torch.logsumexp(s, 0))) <= 1e-4
    for pool, want in zip(pools, before):
        assert torch.equal(pool.cpu(), want)


def _check_tables(lens, past, share, page=16, seed=0, begin=0, short=0, stream=None, null_slots=False):
    """build_page_tables_packed against a loop over the requests; everything that build_page_tables writes too is the same."""
    import random

    from paper_2502_02534_amd import binding as B
    rng = random.Random(seed)
    n = len(lens)
    held_counts = [-(-x // page) + (rng.randrange(3) == 0) for x in past] if past else [0] * n
    had = past or [0] * n
    want = [max(a, b, 0) for a, b in zip(lens, had)]
    need = [max(0, -(-w // page) - h) for w, h in zip(want, held_counts)]
    count = begin + int(min(sum(need), 1 << 20) * share)
    ids = list(range(sum(held_counts) + count))
    rng.shuffle(ids)
    first = _starts(held_counts)
    free = ids[first[-1]:]
    served, running = [], 0
    for k in need:
        running += k
        served.append(k == 0 or running <= len(free) - begin)
    most = (1 << 31) - 1
    asked = [w - h for w, h in zip(want, had)]
    want_indptr = [min(x, most) for x in _starts(asked)]
    slots, taken = [], begin
    for i in range(n):
        mine = ids[first[i]:first[i + 1]]
        if served[i]:
            mine += free[taken:taken + need[i]]
            taken += need[i]
        places = asked[i] if served[i] else min(asked[i], 70000)  # (what is refused may be more than any list holds)
        slots += [mine[t // page] * page + t % page for t in range(had[i], want[i])] if served[i] else [-1] * places
    total = min(sum(asked), len(slots))
    max_pages, max_tokens = sum(held_counts) + count + 5, max(total + 5 - short, 0)
    want_slots = (slots + [-1] * 5)[:max_tokens]
    held_args = (_i32(past), _i32(first), _i32(ids[:first[-1]] or [0])) if past else (None, None, None)
    args = (n, page, _i32(lens), *held_args, _i32(free or [0]), len(free), _i32([begin]) if begin else None, max_pages, max_tokens)
    outs = []
    print(f"packed tables n {n} page {page} share {share} begin {begin} tokens {sum(asked)}", flush=True)
    for packed in (False, True):
        fill = lambda k, t=torch.int32: torch.full((k,), -9, dtype=t, device=DEV)  # noqa: E731
        out = [fill(n + 1), fill(max_pages), fill(n), fill(n + 1)]
        slot_map, end, packed_indptr, packed_lens = fill(max_tokens + 3, torch.int64), fill(1), fill(n + 1), fill(n)
        ws = torch.empty(B.build_page_tables_workspace_size(n), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        if packed:
            B.build_page_tables_packed(*args, *out, None if null_slots else slot_map, end, packed_indptr, packed_lens, ws, stream)
        else:
            B.build_page_tables(*args, *out, slot_map, end, ws, stream)
        torch.cuda.synchronize()
        outs.append(out + [end])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert outs[0][2].tolist() == [w if s else h for w, h, s in zip(want, had, served)]
    assert packed_indptr.tolist() == want_indptr
    assert packed_lens.tolist() == [w if s else 0 for w, s in zip(want, served)]
    assert slot_map.tolist() == ([-9] * (max_tokens + 3) if null_slots else want_slots + [-9] * 3)


@pytest.mark.parametrize("n", [1, 3, 64, 513, 2047, 2048, 2049, 5000])
@pytest.mark.parametrize("share", [0.0, 0.4, 0.999, 1.0])
def test_tables_of_packed_rows(n, share):
    import random
    rng = random.Random(n)
    _check_tables([rng.randrange(0, 60) for _ in range(n)], None, share, seed=n)
    past = [rng.randrange(0, 50) for _ in range(n)]
    _check_tables([x + rng.choice([0, 1, 3, 40]) for x in past], past, share, seed=n + 1, begin=n % 3)


@pytest.mark.parametrize("page", [1, 7, 64, 65536])
def test_tables_of_packed_rows_with_other_pages(page):
    for share in (0.0, 0.7, 1.0):
        _check_tables([0, 1, page, page + 1, 9], [0, 1, 5, 9, 9], share, page=page)


def test_tables_of_packed_rows_at_their_ends():
    _check_tables([30, 50, 1], [16, 0, 1], 0.5, short=20)               # a slot map that is too short is not overrun
    _check_tables([30, 50, 1], [16, 0, 1], 0.5, null_slots=True)
    _check_tables([0, 0, -7], None, 1.0)                                # nothing asked for
    _check_tables([3, 100], [50, 20], 0.0)                              # shorter than what is held
    _check_tables([30, 50, 1], [16, 0, 1], 0.5, stream=torch.cuda.Stream())


@pytest.mark.parametrize("n", [6, 2100])
def test_more_tokens_asked_for_than_32_bits_count(n):
    """Refused, all of them: the count stops at 2^31 - 1 and what comes before has its places."""
    from paper_2502_02534_amd import binding as B
    most = (1 << 31) - 1
    lens = [5, most, 7, most, most, 20] + [0] * (n - 6)
    fill = lambda k, t=torch.int32: torch.full((k,), -9, dtype=t, device=DEV)  # noqa: E731
    ip, px, lo, ni, sm, end, pi, pl = fill(n + 1), fill(4), fill(n), fill(n + 1), fill(50, torch.int64), fill(1), fill(n + 1), fill(n)
    ws = torch.empty(B.build_page_tables_workspace_size(n), dtype=torch.uint8, device=DEV)
    B.build_page_tables_packed(n, 16, _i32(lens), None, None, None, _i32([8, 9]), 2, None, 4, 50, ip, px, lo, ni, sm, end, pi, pl, ws)
    torch.cuda.synchronize()
    assert pi.tolist() == [0, 5] + [most] * (n - 1) and pl.tolist() == [5] + [0] * (n - 1) and lo.tolist() == pl.tolist()
    assert sm.tolist() == [128, 129, 130, 131, 132] + [-1] * 45 and end.tolist() == [1]
