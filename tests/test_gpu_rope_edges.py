"""Rotary positions at the ends of what a call may be: the most rows; a session's tables by the definition, and when they may change."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


def test_as_many_rows_as_a_call_takes(cass):
    """2^31 - 1 rows of one head, in place, the row its position.  Tolerances: a turn as in test_gpu_rope.py (6 x 2^-24 of |a| + |b|, a few 2^-53 of the
    angle), the result rounded to the type (half a step, 2^-25 at least)."""
    rows = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("no room for that many rows")
    x = torch.zeros(rows, 1, 2, dtype=torch.float16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    at = torch.cat([torch.arange(1000), torch.randint(0, rows, (1000,)), torch.arange(rows - 1000, rows)]).unique().cuda()
    x[at] = torch.randn(len(at), 1, 2, generator=g, device="cuda").half()
    before = x[at].double()
    freqs = torch.tensor([0.7, 1.0], dtype=torch.float64, device="cuda")
    geom = cass.RopeGeom(cass.F16, 2, 2, 0, 1, 0, 2, 2, 0, 0, 2, 2, 0, 0)
    cass.cass_rope(geom, freqs, None, rows, x, None, x, None)
    t = at.double() * 0.7
    a, b = before[:, 0, 0], before[:, 0, 1]
    want = torch.stack((a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()), 1)
    tol = (a.abs() + b.abs())[:, None] * (6 * 2.0 ** -24 + t[:, None] * 4 * 2.0 ** -53) + want.abs() * 2.0 ** -11 * (1 + 2.0 ** -10) + 2.0 ** -25
    assert ((x[at][:, 0].double() - want).abs() <= tol).all()


def test_engine_turns_by_other_frequencies_only_while_its_caches_are_empty(cass):
    import dataclasses

    import synth
    from paper_2605_26558_b200 import engine
    shape = dataclasses.replace(synth.TINY, n_layers=1)
    w = synth.model_weights(shape, 5, "cuda")
    w["layers"] = [engine.fuse_layer_weights(lw) for lw in w["layers"]]
    eng = engine.Engine(shape, w, max_seq=128)
    params = cass.RopeParams(shape.head_dim, cass.ROPE_LINEAR, shape.rope_theta, 2.0, 1.0, 4.0, 64.0, 0.0)
    eng.set_rope(params)
    eng.prefill(synth.random_prompt(20, shape.vocab, 4))
    with pytest.raises(cass.CassError) as e:
        eng.set_rope(params)
    assert e.value.code == cass.ERR_INVALID_ARG
    eng.reset()
    eng.set_rope(params)
    eng.close()


@pytest.mark.parametrize("kind", ["none", "linear", "ntk", "bands", "yarn"])
@pytest.mark.parametrize("factor", [2.0, 8.0])
def test_a_session_turns_by_the_definition(cass, kind, factor):
    """q and k of a verification of one token at positions 0 to 8: unscaled, its first row is the unturned one (rounded to 16 bits before the
    rotation), and every row of a scaled session is that one turned by the definition's angle.  Tolerances of test_gpu_rope.py."""
    import dataclasses

    import synth
    import test_gpu_rope
    from paper_2605_26558_b200 import engine
    shape = dataclasses.replace(synth.TINY, n_layers=1)
    w = synth.model_weights(shape, 5, "cuda")
    w["layers"] = [engine.fuse_layer_weights(lw) for lw in w["layers"]]
    eng = engine.Engine(shape, w, max_seq=128)
    rows, d, heads = 9, shape.head_dim, shape.n_q_heads + shape.n_kv_heads
    toks = torch.full((1, rows), 77, device="cuda", dtype=torch.int32)

    def turned():
        eng.reset()
        cass.cass_verify(eng.session, toks, rows - 1, torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, shape.vocab, device="cuda"))
        ptr, _, cols = cass.cass_debug_activation(eng.session, 2)
        o = ptr - eng.mem.data_ptr()
        return eng.mem[o: o + 2 * rows * cols].view(torch.bfloat16).view(rows, -1, d)[:, :heads].clone()

    x = turned()[:1].expand(rows, -1, -1)
    eng.reset()
    which = ("none", "linear", "ntk", "bands", "yarn").index(kind)
    eng.set_rope(cass.RopeParams(d, which, shape.rope_theta, factor, 1.0, 4.0, 64.0, 0.0))
    freqs, gain = test_gpu_rope.frequencies(d, kind, shape.rope_theta, factor, 1.0, 4.0, 64.0)
    test_gpu_rope.check(turned(), x, torch.arange(rows, device="cuda"), freqs, gain, False, 0)
    eng.close()
