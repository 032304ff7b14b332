"""A prompt pass whose requests bring no new tokens does nothing."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("slots", [0, 5])
def test_a_pass_without_tokens(dtype, slots):
    from paper_2502_02534_amd import device as dev
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    held = dev.PageTables(i32(0, 1, 2), i32(3, 1), i32(16, 2), i32(0, 0, 0), None, i32(0))
    t = dev.build_tables(i32(16, 2), i32(0, 2), 4, slots, held=held)
    pools = [torch.randn((4, 2, 16, 64), device=DEV).to(dtype) for _ in range(2)]
    before = [x.clone() for x in pools]
    none = lambda heads: torch.empty((0, heads, 64), dtype=dtype, device=DEV)  # noqa: E731
    run = dev.DevicePrompts(t, none(8), none(2), none(2), *pools, 0, 16)
    run.run()
    torch.cuda.synchronize()
    assert run.out.shape == (0, 8, 64) and run.lse.shape == (0, 8)
    assert all(torch.equal(a, b) for a, b in zip(pools, before))
    assert t.lens.tolist() == [16, 2] and t.page_indices.tolist() == [3, 1, -1, -1]
