"""What build_page_tables_packed refuses on the host (no GPU needed: the pointers are never dereferenced)."""
import os

import pytest

P = 4096          # a pointer, never dereferenced
EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def B():
    from paper_2502_02534_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    binding.load()
    return binding


def _tables(B, n=4, page=16, lens=P, hl=0, hi=0, hp=0, free=P, num_free=10, begin=0, mp=10, mt=10, pi=P, px=P, lo=P, ni=P, sm=P, fe=P,
            ki=P, kl=P, ws=P, size=1 << 20):
    return B.load().build_page_tables_packed(n, page, lens, hl, hi, hp, free, num_free, begin, mp, mt, pi, px, lo, ni, sm, fe, ki, kl,
                                             ws, size, 0)


def test_build_page_tables_packed_refuses(B):
    for name in ("lens", "free", "pi", "px", "lo", "ni", "fe", "ki", "kl"):
        assert _tables(B, **{name: 0}) == EINVAL, name
        assert _tables(B, **{name: P + 1}) == EINVAL, name
    assert _tables(B, n=0) == EINVAL and _tables(B, page=0) == EINVAL and _tables(B, sm=P + 4) == EINVAL and _tables(B, hl=P) == EINVAL
    assert _tables(B, page=65537) == EUNSUPPORTED and _tables(B, n=1 << 31) == EUNSUPPORTED
    assert _tables(B, begin=P, fe=P) == EINVAL
    assert _tables(B, ws=0) == EWORKSPACE and _tables(B, size=8) == EWORKSPACE
    with pytest.raises(B.SpdError, match="build_page_tables_packed"):
        B.build_page_tables_packed(0, 16, None, None, None, None, None, 0, None, 0, 0, None, None, None, None, None, None, None, None, None, 0)
