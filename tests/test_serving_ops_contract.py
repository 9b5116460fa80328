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


def test_evictions_that_keep_more_than_32_bits_of_steps(cass):
    most = 2 ** 31 - 2 ** 16
    p = lambda i: C.c_void_p(AT + (i << 24))  # noqa: E731

    def call(capacity, budget, weight_out=None):
        c = cass.CacheGeom(cass.BF16, 1, 1, 8, capacity, 0, 8, 0)
        return cass.lib.cass_kv_evict(C.byref(c), p(0), p(1), p(2), p(3), budget, 0, 0, None, None, None, weight_out, p(4), p(5), None)

    assert call(2 ** 31 - 1, most + 1) == call(most + 1, 100, p(6)) == cass.ERR_UNSUPPORTED


@pytest.mark.parametrize("lens", [[0], [7], [0, 0], [0, 3]])
def test_an_engine_with_positions_in_its_caches_keeps_its_rotation(cass, monkeypatch, lens):
    from paper_2605_26558_b200 import engine
    calls = []
    monkeypatch.setattr(engine.B, "cass_session_lens", lambda session, batch: lens)
    monkeypatch.setattr(engine.B, "cass_session_set_rope", lambda session, params: calls.append(params))
    eng = object.__new__(engine.Engine)
    eng.session, eng.batch, eng.n_prompt = None, len(lens), 0
    if any(lens):
        with pytest.raises(cass.CassError) as e:
            eng.set_rope("params")
        assert e.value.code == cass.ERR_INVALID_ARG and not calls
    else:
        eng.set_rope("params")
        assert calls == ["params"]
