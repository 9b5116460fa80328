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


def test_tensors_of_other_types_are_refused(cass):
    """A length in torch's own 64-bit integers would be read as two 32-bit ones, 32-bit values as pairs of 16-bit ones.  (Tensors of the host:
    with the right types it is their place that is refused.)"""
    import torch
    i32, f32, f64 = (torch.zeros(8, dtype=t) for t in (torch.int32, torch.float32, torch.float64))
    half, bf = torch.zeros(64, dtype=torch.float16), torch.zeros(64, dtype=torch.bfloat16)
    i64, bits = torch.zeros(8, dtype=torch.int64), torch.zeros(64, dtype=torch.int16)
    cache = cass.CacheGeom(cass.BF16, 1, 1, 32, 2, 64, 32, 32)
    attn = cass.SharedAttn(1, 1, 32, 32, 32, 32, 32, 32, 2, 32, 32, 0.0)
    geom = cass.RopeGeom(cass.F32, 4, 4, 0, 1, 0, 4, 4, 0, 0, 4, 4, 0, 0)

    def refused(call, good, bad):
        """Every argument of `bad` in turn instead of the one of `good`."""
        with pytest.raises(AssertionError):
            call(*good)
        for at, wrong in bad.items():
            for x in wrong:
                with pytest.raises(TypeError, match="tensor of"):
                    call(*good[:at], x, *good[at + 1:])

    refused(cass.cass_rope, [geom, f64, i32, 2, f32, None, f32, None], {1: [f32], 2: [i64, f32], 4: [half, f64], 6: [bf]})
    refused(cass.cass_rope_freqs, [cass.RopeParams(4, 0, 1e4, 1.0, 1.0, 4.0, 64.0, 0.0), f64], {1: [f32]})
    refused(cass.cass_shared_prefix_attention, [cache, attn, bf, bf, bf, bf, bits, i32, bf, f32, f32, f32, f32, 32, i32],
            {2: [half, f32], 3: [half], 6: [half], 7: [i64], 8: [f32], 9: [f64, half], 10: [f64], 11: [bf], 14: [i64]})
    refused(cass.cass_kv_evict, [cache, bf, bits, f32, i32, 1, 0, 0, cache, bf, bf, f32, i32, i32],
            {1: [half], 2: [f32], 3: [f64], 4: [i64], 9: [half], 11: [bf], 12: [i64], 13: [i64]})


def test_an_eviction_of_keys_and_values_in_one_place_is_refused(cass):
    """Both would be moved over one another.  (Read from one place and written to two, they may be the same.)"""
    c, out = (cass.CacheGeom(cass.BF16, 1, 1, 8, n, 0, 8, 0) for n in (100, 50))
    p = lambda i: C.c_void_p(AT + (i << 24))  # noqa: E731
    assert cass.lib.cass_kv_evict(C.byref(c), p(0), p(0), p(2), p(3), 50, 0, 0, None, None, None, None, p(4), p(5), None) == cass.ERR_INVALID_ARG
    assert cass.lib.cass_kv_evict(C.byref(c), p(0), p(1), p(2), p(3), 50, 0, 0, C.byref(out), p(6), p(6), None, p(4), p(5), None) == cass.ERR_INVALID_ARG
