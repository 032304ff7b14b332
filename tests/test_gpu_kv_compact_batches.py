"""`compact_kv` of many sequences, where every workgroup takes all places of its rows or longer stretches of them.  Everything is equal."""
import pytest

import readout_reference as R
from test_gpu_kv_eviction import Cache, run_compact, same

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PAGE = 16


def slots(cache):
    """The slot of every sequence's tokens."""
    at = []
    for b, n in enumerate(cache.lens):
        t = torch.arange(n)
        at.append(cache.pages[int(cache.indptr[b]) + t // PAGE].long() * PAGE + t % PAGE if cache.page else int(cache.indptr[b]) + t)
    return at


def rows(cache, pool):
    """The pool as [slots, heads, channels]."""
    return pool.transpose(1, 2).flatten(0, 1) if cache.page else cache.heads(pool)


def expected(old, new, sources, weights_out):
    k, v, w = rows(new, new.k).clone(), rows(new, new.v).clone(), weights_out.clone()
    ok, ov, frm, to = rows(old, old.k), rows(old, old.v), slots(old), slots(new)
    for b in range(len(old.lens)):
        for j in range(old.hkv):
            s = torch.tensor(sources[b][j], dtype=torch.int64)
            k[to[b][:len(s)], j], v[to[b][:len(s)], j] = ok[frm[b][s], j], ov[frm[b][s], j]
            w[b, j, :len(s)] = old.weights[b, j][s]
            w[b, j, len(s):] = 0
    return k, v, w


def lists(cache, keep, recents, seed=0):
    """`keep` of 8 tokens stay; sequences take the sizes of `recents` in turn, so that some shift places that others read."""
    g = torch.Generator().manual_seed(seed)
    return [[R.kept(torch.rand(max(n, 1), generator=g).tolist(), n, n * keep // 8, 2, recents[b % len(recents)]) for _ in range(cache.hkv)]
            for b, n in enumerate(cache.lens)]


def check(old, new, s, **kw):
    k, v, w = run_compact(old, new, s, **kw)
    ek, ev, ew = expected(old, new, s, old.weights if kw.get("weights_in_place", True) else torch.full_like(old.weights, 7.0))
    assert same(rows(new, k).contiguous(), ek) and same(rows(new, v).contiguous(), ev) and torch.equal(w, ew)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("keep,recents", [(4, [0]), (6, [0, 300, 7, 10 ** 6])])
def test_batches_in_place(dtype, d, page, keep, recents):
    """1024 (sequence, KV head) pairs and more: a workgroup has keys and values of all places, more than it looks at in one go for some."""
    hkv = 4
    c = Cache(dtype, hkv, d, [(i * 37) % 130 for i in range(255)] + [2100, 1500, 1025, 1024], page, seed=d)
    check(c, c, lists(c, keep, recents))


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("recents", [[0], [0, 0, 0, 500]])
@pytest.mark.parametrize("short", [56, 296])
def test_stretches_of_many_rows_in_place(page, recents, short):
    """Fewer pairs, whose stretches are longer than the shortest: several a row, and one."""
    c = Cache("bf16", 2, 64, [(i * 53) % 40 for i in range(short)] + [3000, 2000, 1100, 600], page, seed=3)
    check(c, c, lists(c, 6, recents))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [0, 16])
def test_many_rows_into_other_pages(dtype, page):
    old = Cache(dtype, 2, 64, [(i * 29) % 30 for i in range(1000)] + [2500, 1300], page, seed=1)
    new = Cache(dtype, 2, 64, [n * 7 // 8 for n in old.lens], page, seed=2)
    check(old, new, lists(old, 7, [0, 64]), in_place=False, weights_in_place=False)
