"""`compact_kv` on contiguous tokens in place: pages that a caller hands over for one table and not the other change nothing."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("which", ["neither", "in", "out"])
def test_shift_by_a_few_places(which):
    """Every place is read after others were written: the order of the walk counts."""
    from paper_2502_02534_amd import binding as B
    n, hkv, d, room, shift = 3, 2, 128, 3000, 7
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((n * room, hkv, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    want = [x.clone().view(n, room, hkv, d) for x in (k, v)]
    for x in want:
        x[:, :room - shift] = x[:, shift:].clone()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    source = torch.arange(shift, room, dtype=torch.int32, device=DEV).expand(n, hkv, room - shift).contiguous()
    starts, junk = i32([room * b for b in range(n + 1)]), i32([0])
    desc = B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=hkv, num_kv_heads=hkv, head_dim=d, num_prompts=n, page_size=0)
    B.compact_kv(desc, source, source.stride(0), source.stride(1), i32([room - shift] * n), room - shift, starts, junk if which == "in" else None, k, v,
                 starts, junk if which == "out" else None, k, v, None, None, 0, None)
    torch.cuda.synchronize()
    for x, y in zip((k, v), want):
        assert torch.equal(x.view(n, room, hkv, d), y)
