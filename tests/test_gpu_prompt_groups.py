"""`prompt_attn` of some prompts out of a larger packed batch: the group's starts do not begin at 0, and what lies before and
after its rows belongs to others.  Reference and tolerances are those of tests/test_gpu_prompt_attn.py."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_prompt_attn import DEV, PAGE  # noqa: E402
from test_gpu_prompt_attn_paths import Whole  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, PAGE])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,new,past", [((8, 2), [3, 2, 5, 4], [1500, 900, 700, 20]),      # in parts
                                            ((32, 32), [40, 700, 650, 30], [0, 100, 0, 60])])  # as they are, but for the last group
def test_rows_of_other_prompts_are_left_alone(dtype, page, d, heads, new, past):
    from paper_2502_02534_amd import binding as B
    p = Whole(dtype, *heads, d, new, past, page=page, seed=d)
    ref, mass, ref_lse = p.reference()
    tol, lse_tol = p.tolerance(mass), p.lse_tolerance()
    up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
    q, k, v, pages = up(p.q), up(p.k), up(p.v), up(p.pages)
    starts, lens, kv_starts = up(p.query_indptr), up(p.kv_lens), up(p.kv_indptr)
    for first, last in ((1, 3), (2, 4), (3, 4), (0, 2)):
        print(f"group {dtype} {d} page {page} prompts {first} to {last} of {new}", flush=True)
        desc = B.make_prompt_desc(dtype=B.SPD_F32 if dtype == "f32" else B.SPD_BF16, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=d,
                                  num_prompts=last - first, page_size=page)
        mq, mk = max(new[first:last]), max(p.kv[first:last])
        ws = torch.full((max(B.prompt_attn_workspace_size(desc, p.total, mq, mk), 256),), 255, dtype=torch.uint8, device=DEV)
        out, lse = torch.full_like(q, 7.0), torch.full((p.total, heads[0]), 7.0, device=DEV)
        # the binding hands over addresses: a view that starts at the group's first prompt
        B.prompt_attn(desc, q, k, v, starts[first:], lens[first:], kv_starts[first:], pages, p.total, mq, mk, out, lse, ws)
        torch.cuda.synchronize()
        out, lse = out.cpu(), lse.cpu()
        a, b = int(p.query_indptr[first]), int(p.query_indptr[last])
        assert bool((out[:a] == 7.0).all()) and bool((out[b:] == 7.0).all())
        assert bool((lse[:a] == 7.0).all()) and bool((lse[b:] == 7.0).all())
        assert bool(((out[a:b].double() - ref[a:b]).abs() <= tol[a:b]).all())
        assert bool(((lse[a:b].double() - ref_lse[a:b]).abs() <= lse_tol[a:b]).all())
