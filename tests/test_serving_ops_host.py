"""Refusals and size queries of the serving operators (rotary positions, shared-prefix attention, eviction) that need no GPU: what is
refused here is refused before anything is launched."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def cass():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2605_26558_b200 as m
    return m


AT = 0x7F0000000000                # an aligned address that nothing here reads


def _code(rc):
    return int(rc)


def rope_params(cass, **kw):
    v = dict(rot_dim=64, scaling=cass.ROPE_PLAIN, theta=1e4, factor=2.0, low=1.0, high=4.0, trained_len=4096.0, gain=0.0)
    v.update(kw)
    return cass.RopeParams(*v.values())


@pytest.mark.parametrize("kw", [
    dict(rot_dim=0), dict(rot_dim=63), dict(scaling=5), dict(scaling=-1), dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")),
    dict(scaling=1, factor=0.0), dict(scaling=1, factor=float("nan")), dict(scaling=2, rot_dim=2), dict(scaling=3, low=4.0), dict(scaling=3, low=0.0),
    dict(scaling=4, trained_len=0.0), dict(scaling=4, high=float("inf")), dict(gain=-1.0)])
def test_rope_parameters_that_mean_nothing(cass, kw):
    assert _code(cass.lib.cass_rope_freqs(C.byref(rope_params(cass, **kw)), C.c_void_p(AT), None)) == cass.ERR_INVALID_ARG


def rope_geom(cass, **kw):
    v = dict(dtype=cass.BF16, head_dim=64, rot_dim=64, interleaved=0, n_q_heads=4, n_k_heads=2, q_row=256, q_head=64, k_row=128, k_head=64,
             q_out_row=256, q_out_head=64, k_out_row=128, k_out_head=64)
    v.update(kw)
    return cass.RopeGeom(*v.values())


def call_rope(cass, g, rows=5, q=AT, k=AT + (1 << 20), qo=AT + (2 << 20), ko=AT + (3 << 20), freqs=AT + (4 << 20), pos=0):
    p = lambda x: C.c_void_p(x)  # noqa: E731
    return _code(cass.lib.cass_rope(C.byref(g), p(freqs), p(pos), rows, p(q), p(k), p(qo), p(ko), 0, None))


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(rot_dim=65), dict(rot_dim=66), dict(rot_dim=0), dict(n_q_heads=-1), dict(n_q_heads=0), dict(n_k_heads=0), dict(q_row=-1),
    dict(q_out_row=0), dict(q_out_row=255), dict(q_out_head=63), dict(k_out_row=64, k_out_head=64), dict(k_out_head=-64)])
def test_rope_layouts_that_are_refused(cass, kw):
    assert call_rope(cass, rope_geom(cass, **kw)) == cass.ERR_INVALID_ARG


def test_rope_pointers_that_are_refused(cass):
    g = rope_geom(cass)
    inv = cass.ERR_INVALID_ARG
    assert call_rope(cass, g, q=0) == inv and call_rope(cass, g, ko=0) == inv and call_rope(cass, g, freqs=0) == inv
    assert call_rope(cass, g, q=AT + 1) == inv and call_rope(cass, g, freqs=AT + 4) == inv and call_rope(cass, g, pos=AT + 2) == inv
    assert call_rope(cass, g, rows=-1) == inv
    assert call_rope(cass, rope_geom(cass, q_row=512), qo=AT) == inv                   # in place into another layout
    assert call_rope(cass, rope_geom(cass, n_q_heads=1 << 17, q_out_row=1 << 30)) == cass.ERR_UNSUPPORTED
    assert call_rope(cass, rope_geom(cass, n_q_heads=60000, q_out_row=60000 * 64), rows=1 << 20) == cass.ERR_UNSUPPORTED
    assert call_rope(cass, g, rows=0) == cass.OK                                       # nothing to do
    assert _code(cass.lib.cass_rope(None, C.c_void_p(AT), None, 1, None, None, None, None, 0, None)) == inv


def cache_geom(cass, **kw):
    v = dict(dtype=cass.BF16, n_seq=3, n_kv_heads=2, head_dim=64, capacity=100, seq_stride=12800, pos_stride=128, head_stride=64)
    v.update(kw)
    return cass.CacheGeom(*v.values())


def shared_attn(cass, **kw):
    v = dict(n_q_heads=8, rows=2, q_seq=1024, q_row=512, q_head=64, out_seq=1024, out_row=512, out_head=64, prefix_len=50, prefix_pos_stride=128,
             prefix_head_stride=64, scale=0.0)
    v.update(kw)
    return cass.SharedAttn(*v.values())


BAD_CACHE = [dict(dtype=2), dict(n_seq=0), dict(n_kv_heads=0), dict(capacity=-1), dict(pos_stride=127), dict(pos_stride=64), dict(seq_stride=6400),
             dict(head_stride=0), dict(head_stride=-64), dict(seq_stride=0), dict(head_stride=56)]


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_caches_that_are_refused(cass, kw):
    c, t = cache_geom(cass, **kw), shared_attn(cass)
    assert cass.lib.cass_shared_prefix_scratch_bytes(C.byref(c), C.byref(t), 0) == 0
    p = lambda i: C.c_void_p(AT + (i << 24))  # noqa: E731
    assert _code(cass.lib.cass_kv_evict(C.byref(c), p(0), p(1), p(2), p(3), 50, 0, 0, None, None, None, None, p(4), p(5), None)) == cass.ERR_INVALID_ARG


def test_layouts_that_are_taken(cass):
    size = lambda c, t, w=0: cass.lib.cass_shared_prefix_scratch_bytes(C.byref(c), C.byref(t), w)  # noqa: E731
    plain = size(cache_geom(cass), shared_attn(cass))
    assert plain > 0
    assert size(cache_geom(cass), shared_attn(cass), 1) >= plain + 3 * 8 * 2 * 100 * 4              # scores of every query head and row
    assert size(cache_geom(cass, pos_stride=64, head_stride=6400), shared_attn(cass)) > 0            # heads before positions
    assert size(cache_geom(cass, seq_stride=128, pos_stride=384), shared_attn(cass)) > 0             # positions before sequences
    assert size(cache_geom(cass, n_seq=1, seq_stride=0), shared_attn(cass)) > 0
    assert size(cache_geom(cass, capacity=0, seq_stride=0, pos_stride=0, head_stride=0), shared_attn(cass)) > 0
    for d in (32, 64, 96, 128, 192, 256):
        assert size(cache_geom(cass, head_dim=d, head_stride=d, pos_stride=2 * d, seq_stride=200 * d),
                    shared_attn(cass, q_head=d, q_row=8 * d, q_seq=16 * d, out_head=d, out_row=8 * d, out_seq=16 * d, prefix_head_stride=d,
                                prefix_pos_stride=2 * d)) > 0


@pytest.mark.parametrize("kw,cache", [
    (dict(rows=0), {}), (dict(rows=17), {}), (dict(n_q_heads=7), {}), (dict(n_q_heads=0), {}), (dict(n_q_heads=34), {}), (dict(prefix_len=-1), {}),
    (dict(scale=-1.0), {}), (dict(scale=float("nan")), {}), (dict(scale=float("inf")), {}), (dict(q_row=511), {}), (dict(q_head=-64), {}),
    (dict(out_row=64), {}), (dict(out_seq=512), {}), (dict(prefix_pos_stride=4), {}), ({}, dict(head_dim=80, head_stride=80, pos_stride=160, seq_stride=16000)),
    ({}, dict(head_dim=16)), ({}, dict(n_seq=1025))])
def test_attention_that_is_refused(cass, kw, cache):
    assert cass.lib.cass_shared_prefix_scratch_bytes(C.byref(cache_geom(cass, **cache)), C.byref(shared_attn(cass, **kw)), 0) == 0
    with pytest.raises(cass.CassError):
        cass.cass_shared_prefix_scratch_bytes(cache_geom(cass, **cache), shared_attn(cass, **kw))


def test_attention_pointers_that_are_refused(cass):
    c, t = cache_geom(cass), shared_attn(cass)
    need = cass.lib.cass_shared_prefix_scratch_bytes(C.byref(c), C.byref(t), 1)
    names = ("q", "kp", "vp", "kc", "vc", "lens", "out", "lse", "w_in", "w_out", "scratch")
    base = {n: AT + (i << 24) for i, n in enumerate(names)}

    def call(cache=c, attn=t, nbytes=need, status=AT + (20 << 24), **kw):
        v = dict(base, **kw)
        p = [C.c_void_p(v[n]) for n in names]
        return _code(cass.lib.cass_shared_prefix_attention(C.byref(cache), C.byref(attn), *p, C.c_size_t(nbytes), C.c_void_p(status), None))

    for n in ("q", "kp", "vp", "kc", "vc", "lens", "out", "scratch", "w_out"):          # w_in without w_out
        assert call(**{n: 0}) == cass.ERR_INVALID_ARG, n
    for n in ("q", "kp", "vp", "kc", "vc", "out", "scratch"):
        assert call(**{n: base[n] + 8}) == cass.ERR_INVALID_ARG, n
    for n in ("lens", "lse", "w_in", "w_out"):
        assert call(**{n: base[n] + 2}) == cass.ERR_INVALID_ARG, n
    assert call(status=0) == cass.ERR_INVALID_ARG
    assert call(nbytes=need - 1) == cass.ERR_CAPACITY
    assert call(cache=cache_geom(cass, capacity=0)) == cass.ERR_INVALID_ARG              # weights of no positions


def test_evictions_that_are_refused(cass):
    c = cache_geom(cass)
    names = ("k", "v", "w", "lens", "ko", "vo", "wo", "kept", "new")
    base = {n: AT + (i << 24) for i, n in enumerate(names)}

    def call(budget=50, first=4, last=8, cache=c, out=None, **kw):
        v = dict(base, ko=0, vo=0) if out is None else dict(base)
        v.update(kw)
        p = {n: C.c_void_p(v[n]) for n in names}
        return _code(cass.lib.cass_kv_evict(C.byref(cache), p["k"], p["v"], p["w"], p["lens"], budget, first, last,
                                            C.byref(out) if out is not None else None, p["ko"], p["vo"], p["wo"], p["kept"], p["new"], None))

    inv = cass.ERR_INVALID_ARG
    for n in ("k", "v", "w", "lens", "kept", "new"):
        assert call(**{n: 0}) == inv, n
    assert call(k=AT + 8) == inv and call(kept=AT + 2) == inv and call(wo=AT + 2) == inv
    for b, f, l in ((0, 0, 0), (101, 0, 0), (50, -1, 0), (50, 0, -1), (50, 51, 0), (50, 25, 26), (50, 2147483647, 2147483647)):
        assert call(budget=b, first=f, last=l) == inv, (b, f, l)
    small = cache_geom(cass, capacity=50)
    assert call(out=small, ko=0) == inv and call(out=small, vo=0) == inv and call(ko=AT) == inv
    assert call(out=small, ko=base["k"]) == inv and call(out=small, vo=base["k"]) == inv
    assert call(out=cache_geom(cass, capacity=49)) == inv
    for kw in (dict(dtype=1), dict(n_seq=2), dict(n_kv_heads=1), dict(head_dim=32)):
        assert call(out=cache_geom(cass, capacity=50, **kw)) == inv, kw
    assert call(out=small, wo=base["w"]) == inv                                          # weights in place, the cache not
    assert call(cache=cache_geom(cass, head_dim=60)) == cass.ERR_UNSUPPORTED
    assert call(cache=cache_geom(cass, head_dim=520, head_stride=520, pos_stride=1040, seq_stride=104000)) == cass.ERR_UNSUPPORTED
