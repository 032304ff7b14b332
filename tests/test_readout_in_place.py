"""`compact_kv` in place: told from the tables that the call uses.  Contiguous tokens have no pages, so what is handed over for them does not
count (no GPU needed: the pointers are never dereferenced)."""
import ctypes
import os

import pytest

P = 4096          # a pointer, never dereferenced
EINVAL = 1


@pytest.fixture(scope="module")
def B():
    from paper_2502_02534_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    binding.load()
    return binding


@pytest.mark.parametrize("kp,op", [(0, 0), (P, P), (P, 2 * P), (0, P), (P, 0)])
def test_pages_of_contiguous_tokens_do_not_count(B, kp, op):
    """Keys in place and values not: refused, whatever the pages are."""
    desc = B.make_prompt_desc(dtype=B.SPD_BF16, num_q_heads=8, num_kv_heads=8, head_dim=64, num_prompts=4, page_size=0)
    assert B.load().compact_kv(ctypes.byref(desc), P, 1000, 500, P, 500, P, kp, 3 * P, 4 * P, P, op, 3 * P, 5 * P, 0, 0, 0, 0, 0) == EINVAL
