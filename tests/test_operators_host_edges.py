"""Arguments at the edges of the operators around the cache: answered or refused on the host (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def hb():
    import __graft_entry__ as ge
    ge.build()
    import paper_2504_09261_b200 as pkg
    return pkg


@pytest.mark.parametrize("norm,eps,refused", [(2, 1e-40, True), (2, 2.0 ** -149, True), (2, 2.0 ** -126, False), (1, 1e-40, False)])
def test_an_eps_without_a_reciprocal_is_refused(hb, norm, eps, refused):
    from paper_2504_09261_b200 import binding as bd
    none = bd.HackStrides()
    args = bd.HackQkvArgs(0, 0, 1, 2, 0, 0, 64, norm, eps, 0, 0, *([none] * 6))       # (no tokens: nothing else is looked at)
    assert bd.lib.hack_qk_norm_rope(None, C.addressof(args), *([None] * 12)) == (1 if refused else 0)
    assert not refused or "reciprocal" in hb.hack_last_error()
