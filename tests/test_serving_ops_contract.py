"""What the serving operators' contract allows or refuses beyond test_serving_ops_host.py; no GPU: nothing here is launched."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def cass():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2605_26558_b200 as m
    return m


AT = 0x7F0000000000                # an aligned address that nothing here reads


@pytest.mark.parametrize("nq,nk", [(4, 2), (4, 0), (0, 2)])
def test_a_rotation_of_no_rows_does_nothing(cass, nq, nk):
    """Tensors without rows have no address."""
    g = cass.RopeGeom(cass.BF16, 64, 64, 0, nq, nk, nq * 64, 64, nk * 64, 64, nq * 64, 64, nk * 64, 64)
    assert cass.lib.cass_rope(C.byref(g), C.c_void_p(AT), None, 0, None, None, None, None, 0, None) == cass.OK
    assert cass.lib.cass_rope(C.byref(g), C.c_void_p(AT), None, 1, None, None, None, None, 0, None) == cass.ERR_INVALID_ARG
    g.n_q_heads = g.n_k_heads = 0
    assert cass.lib.cass_rope(C.byref(g), C.c_void_p(AT), None, 0, None, None, None, None, 0, None) == cass.ERR_INVALID_ARG
