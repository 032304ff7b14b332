"""Requests that hold nothing yet, by tables that were built for nothing."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("n", [3, 2100])
def test_tables_that_grow_from_no_pages(n):
    from paper_2502_02534_amd import device as dev
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    free = torch.arange(100, 100 + n, dtype=torch.int32, device=DEV)
    nothing = dev.build_tables(i32([0] * n), free, 0)
    assert nothing.page_indices.numel() == 0 and nothing.lens.tolist() == [0] * n
    t = dev.build_tables(i32([1 + i % 16 for i in range(n)]), free, n, 16 * n, held=nothing, free_begin=nothing.free_end)
    torch.cuda.synchronize()
    assert t.page_indices.tolist() == list(range(100, 100 + n)) and t.free_end.tolist() == [n]
    want = [(100 + i) * 16 + k for i in range(n) for k in range(1 + i % 16)]
    assert t.slots[:len(want)].tolist() == want and bool((t.slots[len(want):] == -1).all())
