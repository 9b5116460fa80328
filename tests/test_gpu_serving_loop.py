"""The serving operators together, as a decode loop uses them: keys rotated into the caches, attention behind a shared prefix with the
weights summed, eviction when a cache is full, attention over what stayed; and scaled rotary positions through an engine."""
import dataclasses
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("graph", [False, True])
def test_decode_with_eviction(cass, dtype, graph):
    """Twelve steps of five sequences over a budget of 20 positions in caches of 26 behind 150 shared positions; every step against the
    definition in 64 bits on the same caches, every eviction against a plain selection by the same sums."""
    b, nq, nk, d, prefix, cap, budget, first, last, rows = 5, 8, 2, 64, 150, 26, 20, 1, 4, 2
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    half = torch.finfo(dtype).eps / 2
    kind = cass.BF16 if dtype == torch.bfloat16 else cass.F16
    kp, vp = rnd(prefix, nk, d).to(dtype), rnd(prefix, nk, d).to(dtype)
    kc, vc = (torch.zeros(b, cap, nk, d, dtype=dtype, device="cuda") for _ in range(2))
    w = torch.zeros(b, nk, cap, device="cuda")
    lens, kept = torch.zeros(b, dtype=torch.int32, device="cuda"), torch.zeros(b, nk, budget, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    freqs = torch.zeros(d // 2 + 1, dtype=torch.float64, device="cuda")
    cass.cass_rope_freqs(cass.RopeParams(d, cass.ROPE_BANDS, 1e4, 8.0, 1.0, 4.0, 64.0, 0.0), freqs)
    qkv = torch.zeros(b * rows, nq + 2 * nk, d, dtype=dtype, device="cuda")
    q, k = torch.zeros(b, rows, nq, d, dtype=dtype, device="cuda"), torch.zeros(b * rows, nk, d, dtype=dtype, device="cuda")
    pos, out, lse = torch.zeros(b * rows, dtype=torch.int32, device="cuda"), torch.zeros_like(q), torch.zeros(b, rows, nq, device="cuda")
    rope = cass.RopeGeom(kind, d, d, 0, nq, nk, qkv.stride(0), d, qkv.stride(0), d, nq * d, d, nk * d, d)
    cache = cass.CacheGeom(kind, b, nk, d, cap, *kc.stride()[:3])
    attn = cass.SharedAttn(nq, rows, *q.stride()[:3], *out.stride()[:3], prefix, kp.stride(0), kp.stride(1), 0.0)
    scratch = torch.zeros(cass.cass_shared_prefix_scratch_bytes(cache, attn, True), dtype=torch.uint8, device="cuda")
    seqs = torch.arange(b, device="cuda").repeat_interleave(rows)
    at = torch.arange(rows, device="cuda").repeat(b)

    def step():
        cass.cass_rope(rope, freqs, pos, b * rows, qkv.data_ptr(), qkv[:, nq:].data_ptr(), q, k)
        index = (seqs, lens.long()[seqs] + at)
        kc.index_put_(index, k)
        vc.index_put_(index, qkv[:, nq + nk:])
        lens.add_(rows)
        cass.cass_shared_prefix_attention(cache, attn, q, kp, vp, kc, vc, lens, out, lse, w, w, scratch, scratch.numel(), status)

    def evict():
        cass.cass_kv_evict(cache, kc, vc, w, lens, budget, first, last, None, None, None, w, kept, lens)

    run_step, run_evict = step, evict
    if graph:
        graphs = []
        for f in (step, evict):
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                f()
            torch.cuda.current_stream().wait_stream(side)
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr):
                f()
            graphs.append(gr)
        run_step, run_evict = graphs[0].replay, graphs[1].replay
        for t in (kc, vc, w, lens):
            t.zero_()
    true_pos = torch.full((b,), prefix, device="cuda")
    for n in range(12):
        qkv.copy_(rnd(*qkv.shape))
        pos.copy_(true_pos[seqs] + at)
        true_pos += rows
        before = w.double().clone()
        run_step()
        assert int(status.item()) == 0
        for i in range(b):
            for h in range(nk):
                total = before[i, h].clone()
                for r in range(rows):
                    end = int(lens[i]) - (rows - 1 - r)
                    kk, vv = torch.cat((kp[:, h], kc[i, :end, h])).double(), torch.cat((vp[:, h], vc[i, :end, h])).double()
                    s = q[i, r, h * 4:h * 4 + 4].double() @ kk.T / math.sqrt(d)
                    p = torch.softmax(s, 1)
                    size = p @ vv.abs()
                    # probabilities rounded to the type, scores and sums in 32 bits (below 2^-13 of them together), the output rounded
                    assert ((out[i, r, h * 4:h * 4 + 4].double() - p @ vv).abs() <= size * (half + 2.0 ** -13) + (p @ vv).abs() * half * 1.01 + 2.0 ** -25).all()
                    total[:end] += p[:, prefix:].sum(0)
                assert torch.allclose(w[i, h].double(), total, rtol=2.0 ** -13, atol=0)
        if int(lens[0]) + rows > cap:
            state = [t.clone() for t in (kc, vc, w)]
            length = int(lens[0])
            run_evict()
            for i in range(b):
                assert int(lens[i]) == budget
                for h in range(nk):
                    row = state[2][i, h].tolist()
                    mid = sorted(range(first, length - last), key=lambda j: (-row[j], j))[: budget - first - last]
                    want = sorted(list(range(first)) + mid + list(range(length - last, length)))
                    assert kept[i, h].tolist() == want
                    assert torch.equal(kc[i, :budget, h], state[0][i, want, h]) and torch.equal(vc[i, :budget, h], state[1][i, want, h])
                    assert torch.equal(w[i, h, :budget], state[2][i, h, want]) and (w[i, h, budget:] == 0).all()


def test_rotated_keys_move_under_their_positions(cass):
    """Keys turned back and on again (two calls, one of them transposed) score as keys rotated at the new position: what a cache needs
    that moves its positions."""
    d, rows, nk = 64, 40, 2
    freqs = torch.zeros(d // 2 + 1, dtype=torch.float64, device="cuda")
    cass.cass_rope_freqs(cass.RopeParams(d, cass.ROPE_PLAIN, 1e4, 1.0, 1.0, 4.0, 64.0, 0.0), freqs)
    x = torch.randn(rows, nk, d, device="cuda")
    geom = cass.RopeGeom(cass.F32, d, d, 0, 0, nk, 0, 0, nk * d, d, 0, 0, nk * d, d)
    old, new = (torch.randint(0, 5000, (rows,), device="cuda", dtype=torch.int32) for _ in range(2))
    a, c, want = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    cass.cass_rope(geom, freqs, old, rows, None, x, None, a)
    cass.cass_rope(geom, freqs, old, rows, None, a, None, c, 1)
    cass.cass_rope(geom, freqs, new, rows, None, c, None, c)
    cass.cass_rope(geom, freqs, new, rows, None, x, None, want)
    # three rotations after another, each off by 6 x 2^-24 of |a| + |b| <= 2 max
    assert (c - want).abs().max().item() <= 4 * 6 * 2.0 ** -24 * 2 * x.abs().max().item()


def test_engine_with_scaled_positions(cass):
    """Prefill, draft and verification turn by the same scaled tables: the speculative stream equals plain greedy decoding."""
    import synth
    from paper_2605_26558_b200 import engine
    shape = dataclasses.replace(synth.TINY, n_layers=2)
    w = synth.model_weights(shape, 3, "cuda")
    w["layers"] = [engine.fuse_layer_weights(lw) for lw in w["layers"]]
    prompt = synth.random_prompt(40, shape.vocab, 4)

    def stream(gamma):
        eng = engine.Engine(shape, w, max_seq=256, gamma_max=4)
        eng.set_rope(cass.RopeParams(shape.head_dim, cass.ROPE_YARN, shape.rope_theta, 4.0, 1.0, 32.0, 64.0, 0.0))
        first = eng.prefill(prompt, calibrate=True)
        eng.encode_weights(eng.calib_norms())
        eng.build_kv_codebook()
        toks, _ = eng.generate(24, gamma)
        status = eng.status()[0]
        eng.close()
        assert status == 0
        return [first] + toks[:24]

    assert stream(0) == stream(3)
