"""`compact_kv` moves a weight only with its token: places whose source lies past the sequence's table, or that lie past their own,
keep theirs.  Everything is moved or left, so everything is equal."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PAGE = 16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("pairs", [2, 1100])
def test_weights_stay_with_their_tokens(page, in_place, pairs):
    """Sequences of 48 places, of which a table holds 32 (the out table 16): sources up to 31 are there, and weights for 48."""
    from paper_2502_02534_amd import binding as B
    hkv, d, n, stride = 2, 64, pairs // 2, 48
    g = torch.Generator().manual_seed(pairs)
    desc = B.make_prompt_desc(dtype=B.SPD_F32, num_q_heads=hkv, num_kv_heads=hkv, head_dim=d, num_prompts=n, page_size=page)
    shape = lambda pages: (n * pages, hkv, PAGE, d) if page else (n * pages * PAGE, hkv, d)  # noqa: E731
    k, v = torch.randn(shape(2), generator=g), torch.randn(shape(2), generator=g)
    room = 32 if in_place else 16
    ko, vo = (k, v) if in_place else (torch.randn(shape(1), generator=g), torch.randn(shape(1), generator=g))
    w = torch.rand((n, hkv, stride), generator=g)
    wo = w if in_place else torch.rand((n, hkv, stride), generator=g)
    # place i: i itself, one that is there, one past the table, one below it
    source = torch.empty((n, hkv, 24), dtype=torch.int32)
    for i in range(24):
        source[:, :, i] = [i, 24 + i // 4, 32 + i // 3, i - 1][i % 4]
    per = 1 if page else PAGE
    at = lambda pool, b, t, j, pages: pool[b * pages + t // PAGE, j, t % PAGE] if page else pool[b * pages * PAGE + t, j]  # noqa: E731
    want = [x.clone() for x in (ko, vo, wo)]
    for b in (0, n // 2, n - 1):
        for j in range(hkv):
            for i in range(24):
                src = int(source[b, j, i])
                if src >= i and src < 32 and i < room:
                    at(want[0], b, i, j, room // PAGE).copy_(at(k, b, src, j, 2))
                    at(want[1], b, i, j, room // PAGE).copy_(at(v, b, src, j, 2))
                    want[2][b, j, i] = w[b, j, src]
            want[2][b, j, 24:] = 0
    ki, oi = i32([2 * per * b for b in range(n + 1)]), i32([room // PAGE * per * b for b in range(n + 1)])
    kp, op = (i32(list(range(n * 2))), i32(list(range(n * room // PAGE)))) if page else (None, None)
    if in_place:
        oi, op = ki, kp
    kd, vd, wd = k.to(DEV), v.to(DEV), w.to(DEV)
    kod, vod, wod = (kd, vd, wd) if in_place else (ko.to(DEV), vo.to(DEV), wo.to(DEV))
    sd = source.to(DEV)
    B.compact_kv(desc, sd, sd.stride(0), sd.stride(1), i32([24] * n), 24, ki, kp, kd, vd, oi, op, kod, vod, wd, wod, stride, None)
    torch.cuda.synchronize()
    got = [x.cpu() for x in (kod, vod, wod)]
    rows = room // PAGE * per
    for b in (0, n // 2, n - 1):
        assert torch.equal(got[0][b * rows:(b + 1) * rows], want[0][b * rows:(b + 1) * rows])
        assert torch.equal(got[1][b * rows:(b + 1) * rows], want[1][b * rows:(b + 1) * rows])
        assert torch.equal(got[2][b], want[2][b]), b
