"""`device.build_tables` on another stream than the current one: what it allocates belongs to that stream, so that nothing the
current stream allocates meanwhile lies in memory that its launches still write and read."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _requests(n, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, 90, (n,), generator=g).to(torch.int32)
    pages = int(((lens + 15) // 16).sum())
    free = torch.randperm(pages + 9, generator=g).to(torch.int32)
    return lens.to(DEV), free.to(DEV), pages + 3, int(lens.sum()) + 3


def _all(t):
    return [x.clone() for x in (t.page_indptr, t.page_indices, t.lens, t.new_indptr, t.slots, t.free_end)]


@pytest.mark.parametrize("n", [5, 3000])  # one launch, and two that share the workspace
@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_memory_of_a_call_on_another_stream(n, kind, monkeypatch):
    from paper_2502_02534_amd import binding as B
    from paper_2502_02534_amd import device as D
    lens, free, max_pages, max_tokens = _requests(n, n)
    want = _all(D.build_tables(lens, free, max_pages, max_tokens))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    seen = []
    for name in ("build_page_tables", "build_page_tables_packed"):
        monkeypatch.setattr(B, name, lambda *a, call=getattr(B, name): (seen.append(a[-2]), call(*a))[1])
    x = torch.randn((2048, 2048), device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x = torch.tanh(x @ x)  # the side stream is busy for a while
    t = D.build_tables(lens, free, max_pages, max_tokens, stream=side if kind == "stream" else side.cuda_stream)
    first, size = seen[0].data_ptr(), seen[0].numel()
    seen.clear()
    # the current stream goes on: none of its memory is the workspace's
    got = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(8)]
    assert all(a.data_ptr() + a.numel() <= first or a.data_ptr() >= first + size for a in got)
    side.synchronize()
    print(f"tables on a {kind} of their own, {n} requests", flush=True)
    for a, b in zip(_all(t), want):
        assert torch.equal(a, b)


def test_the_default_stream_s_handle():
    from paper_2502_02534_amd import device as D
    lens, free, max_pages, max_tokens = _requests(4, 1)
    torch.cuda.synchronize()
    a = _all(D.build_tables(lens, free, max_pages, max_tokens, stream=0))
    torch.cuda.synchronize()
    for x, y in zip(a, _all(D.build_tables(lens, free, max_pages, max_tokens))):
        assert torch.equal(x, y)
