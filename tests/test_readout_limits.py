"""The operators on a step's softmaxes: calls that no kernel could answer rightly are refused on the host (no GPU needed: the pointers
are never dereferenced)."""
import os

import pytest

P = 4096          # a pointer, never dereferenced
EINVAL, EUNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def B():
    from paper_2502_02534_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    binding.load()
    return binding


def _select(B, seqs=4, heads=2, lens=P, new=2 * P):
    return B.load().select_kv_tokens(P, 40000, seqs, heads, lens, 40000, 0, 500, 4, 32, P, 500, new, 0, 0, 0)


def test_a_launch_counts_its_threads_in_32_bits(B):
    """2^22 rows of 1024 threads are one thread too many."""
    assert _select(B, seqs=1 << 22, heads=1) == EUNSUPPORTED and _select(B, seqs=1 << 21, heads=2) == EUNSUPPORTED
    assert B.select_kv_tokens_workspace_size(1 << 22, 1, 40000) == 0 and B.select_kv_tokens_workspace_size((1 << 22) - 1, 1, 40000) > 0


@pytest.mark.parametrize("heads", [2, 8])
def test_new_lengths_do_not_replace_those_still_read(B, heads):
    """A sequence's first head writes its new length while the others still read the old one."""
    assert _select(B, heads=heads, lens=P, new=P) == EINVAL
