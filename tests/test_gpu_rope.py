"""Rotary positions (cass_rope, cass_rope_freqs, cass_session_set_rope) against the definition in 64 bits.

Tolerances.  A sine or cosine of the kernel is off by at most 3 x 2^-24: the quarter-turn remainder rounded to 32 bits (2^-27 of a
half turn, 2^-25 rad), sincospif (one unit) and the factor (one rounding).  Two products and a sum of them add 2 x 2^-24 of |a| + |b|.
The angle in 64 bits is off by a few 2^-53 of itself.  A result in fewer bits adds half a step, eps / 2 of it."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {torch.bfloat16: "BF16", torch.float16: "F16", torch.float32: "F32"}


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


def frequencies(rot, kind, theta, s=4.0, low=1.0, high=4.0, trained=4096.0):
    """The definition, pair by pair."""
    out = []
    for j in range(rot // 2):
        t = theta * s ** (rot / (rot - 2)) if kind == "ntk" else theta
        f = t ** (-2 * j / rot)
        if kind == "linear":
            f /= s
        elif kind == "bands":
            u = trained * f / (2 * math.pi)
            m = min(max((u - low) / (high - low), 0), 1)
            f = m * f + (1 - m) * f / s
        elif kind == "yarn":
            c = lambda u: rot * math.log(trained / (2 * math.pi * u)) / (2 * math.log(theta))  # noqa: E731
            a, b = max(math.floor(c(high)), 0), min(math.ceil(c(low)), rot - 1)
            m = min(max((j - a) / max(b - a, 0.001), 0), 1)
            f = m * f / s + (1 - m) * f
        out.append(f)
    return torch.tensor(out, dtype=torch.float64), (0.1 * math.log(s) + 1 if kind == "yarn" and s > 1 else 1.0)


def device_freqs(cass, rot, kind, theta=1e4, s=4.0, low=1.0, high=4.0, trained=4096.0, gain=0.0):
    f = torch.full((rot // 2 + 1,), -1.0, dtype=torch.float64, device="cuda")
    kinds = ("none", "linear", "ntk", "bands", "yarn")
    cass.cass_rope_freqs(cass.RopeParams(rot, kinds.index(kind), theta, s, low, high, trained, gain), f)
    return f


@pytest.mark.parametrize("kind", ["none", "linear", "ntk", "bands", "yarn"])
@pytest.mark.parametrize("rot,theta,s", [(64, 1e4, 4.0), (128, 5e5, 8.0), (128, 5e5, 0.5), (34, 1e4, 2.0), (600, 1e6, 40.0)])
def test_frequencies(cass, kind, rot, theta, s):
    want, gain = frequencies(rot, kind, theta, s)
    got = device_freqs(cass, rot, kind, theta, s).cpu()
    # powers of exponents up to ln(theta^2) = 28: their rounding times that, and a unit or two of pow and log on either side
    assert torch.allclose(got[:-1], want, rtol=64 * 2.0 ** -52, atol=0)
    assert abs(got[-1].item() - gain) <= 1e-15
    assert device_freqs(cass, rot, kind, theta, s, gain=1.25)[-1].item() == 1.25


def reference(x, pos, freqs, gain, interleaved, transpose):
    rot = 2 * len(freqs)
    t = pos.double()[:, None, None] * freqs
    c, s = t.cos() * gain, t.sin() * gain * (-1 if transpose else 1)
    y = x.double().clone()
    if interleaved:
        a, b = y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        a, b = y[..., : rot // 2].clone(), y[..., rot // 2: rot].clone()
        y[..., : rot // 2], y[..., rot // 2: rot] = a * c - b * s, a * s + b * c
    size = torch.zeros_like(y)
    pair = (a.abs() + b.abs()) * gain
    if interleaved:
        size[..., 0:rot:2] = size[..., 1:rot:2] = pair
    else:
        size[..., : rot // 2] = size[..., rot // 2: rot] = pair
    return y, size, t.abs().amax().item()


def check(got, x, pos, freqs, gain, interleaved, transpose):
    y, size, far = reference(x, pos, freqs.to(x.device), gain, interleaved, transpose)
    half = torch.finfo(got.dtype).eps / 2 if got.dtype != torch.float32 else 2.0 ** -24
    tol = size * (6 * 2.0 ** -24 + far * 4 * 2.0 ** -53) + y.abs() * half * (1 + 2.0 ** -10)
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25                              # half a step of its smallest numbers
    bad = (got.double() - y).abs() > tol
    assert not bad.any(), (int(bad.sum()), (got.double() - y).abs().max().item())
    rot = 2 * len(freqs)
    assert torch.equal(got[..., rot:], x[..., rot:])


def geom(cass, q, k, qo, ko, rot, interleaved):
    st = lambda t: (t.stride(0), t.stride(1)) if t is not None else (0, 0)  # noqa: E731
    some = q if q is not None else k
    return cass.RopeGeom(getattr(cass, TYPES[some.dtype]), some.shape[2], rot, int(interleaved), q.shape[1] if q is not None else 0,
                         k.shape[1] if k is not None else 0, *st(q), *st(k), *st(qo), *st(ko))


def rope(cass, q, k, qo, ko, freqs, pos, rot, interleaved, transpose=0, stream=None):
    at = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    some = q if q is not None else k
    cass.cass_rope(geom(cass, q, k, qo, ko, rot, interleaved), freqs, pos, some.shape[0], at(q), at(k), at(qo), at(ko), transpose, stream)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("nq,nk,d,rot", [(4, 2, 64, 64), (32, 8, 128, 128), (40, 8, 128, 64), (5, 1, 80, 32), (3, 3, 96, 96), (1, 0, 8, 2), (0, 1, 7, 6),
                                         (2, 1, 256, 250), (1, 1, 1200, 1100), (7, 2, 64, 48), (2, 2, 64, 6)])
def test_against_the_definition(cass, dtype, interleaved, nq, nk, d, rot):
    for rows in (1, 3, 67, 1000):
        g = torch.Generator(device="cuda").manual_seed(rows + rot)
        q, k = (torch.randn(rows, n, d, generator=g, device="cuda").to(dtype) if n else None for n in (nq, nk))
        pos = torch.randint(0, 200000, (rows,), generator=g, device="cuda", dtype=torch.int32)
        kind = ("none", "linear", "bands", "yarn")[rows % 4]
        freqs = device_freqs(cass, rot, kind)
        want, gain = frequencies(rot, kind, 1e4)
        qo, ko = (torch.full_like(t, 7.0) if t is not None else None for t in (q, k))
        for transpose in (0, 1):
            rope(cass, q, k, qo, ko, freqs, pos, rot, interleaved, transpose)
            for x, y in ((q, qo), (k, ko)):
                if x is not None:
                    check(y, x, pos, want, gain, interleaved, transpose)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts_in_place_and_guards(cass, dtype, interleaved):
    """q and k inside packed rows, heads before rows, places off 16-byte boundaries; in place; nothing around them is touched."""
    rows, nq, nk, d, rot = 37, 4, 2, 64, 48
    g = torch.Generator(device="cuda").manual_seed(1)
    pos = torch.randint(-5000, 5000, (rows,), generator=g, device="cuda", dtype=torch.int32)
    freqs, want = device_freqs(cass, rot, "none"), frequencies(rot, "none", 1e4)[0]
    for off in (0, 1, 8):
        flat = torch.randn(off + rows * (nq + 2 * nk) * d + 8, generator=g, device="cuda").to(dtype)
        before = flat.clone()
        qkv = flat[off: off + rows * (nq + 2 * nk) * d].view(rows, nq + 2 * nk, d)
        q, k = qkv[:, :nq], qkv[:, nq: nq + nk]
        q0, k0 = q.clone(), k.clone()
        qo = torch.full((nq, rows, d), 5.0, dtype=dtype, device="cuda").transpose(0, 1)         # [head][row][dim] in memory
        ko = torch.full((rows, nk, d + 8), 5.0, dtype=dtype, device="cuda")
        rope(cass, q, k, qo, ko[..., :d], freqs, pos, rot, interleaved)
        assert torch.equal(flat, before)
        check(qo, q0, pos, want, 1.0, interleaved, 0)
        check(ko[..., :d], k0, pos, want, 1.0, interleaved, 0)
        assert (ko[..., d:] == 5.0).all()
        rope(cass, q, k, q, k, freqs, pos, rot, interleaved)                                     # in place: the same bits
        assert torch.equal(q, qo) and torch.equal(k, ko[..., :d])
        rest = flat.clone()
        rest[off: off + rows * (nq + 2 * nk) * d].view(rows, -1, d)[:, : nq + nk] = before[off: off + rows * (nq + 2 * nk) * d].view(rows, -1, d)[:, : nq + nk]
        assert torch.equal(rest, before)


def test_far_positions_and_positions_by_row(cass):
    d = 128
    freqs, want = device_freqs(cass, d, "none", 5e5), frequencies(d, "none", 5e5)[0]
    x = torch.randn(6, 2, d, device="cuda")
    y = torch.empty_like(x)
    pos = torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9, 131071], dtype=torch.int32, device="cuda")
    rope(cass, x, None, y, None, freqs, pos, d, False)
    check(y, x, pos, want, 1.0, False, 0)
    z = torch.empty_like(x)
    rope(cass, x, None, y, None, freqs, None, d, False)
    rope(cass, x, None, z, None, freqs, torch.arange(6, dtype=torch.int32, device="cuda"), d, False)
    assert torch.equal(y, z)
    rope(cass, x, None, y, None, freqs, torch.zeros(6, dtype=torch.int32, device="cuda"), d, False)
    assert torch.equal(y, x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(cass, interleaved):
    """The transposed call is the gradient: against the formula's (autograd in 64 bits), against differences, and the pairing <R x, g> = <x, R' g>."""
    rows, n, d, rot = 9, 3, 64, 32
    freqs, (want, gain) = device_freqs(cass, rot, "yarn"), frequencies(rot, "yarn", 1e4)
    pos = torch.arange(100, 100 + rows, dtype=torch.int32, device="cuda")
    x, g = torch.randn(rows, n, d, device="cuda"), torch.randn(rows, n, d, device="cuda")
    gx = torch.empty_like(x)
    rope(cass, g, None, gx, None, freqs, pos, rot, interleaved, 1)
    x64 = x.double().requires_grad_()
    t = pos.double()[:, None, None] * want.cuda()
    c, s = t.cos() * gain, t.sin() * gain
    a, b = (x64[..., 0:rot:2], x64[..., 1:rot:2]) if interleaved else (x64[..., : rot // 2], x64[..., rot // 2: rot])
    parts = (a * c - b * s, a * s + b * c)
    turned = torch.stack(parts, -1).flatten(-2) if interleaved else torch.cat(parts, -1)
    torch.cat((turned, x64[..., rot:]), -1).backward(g.double())
    check(gx, g, pos, want, gain, interleaved, 1)
    assert torch.allclose(gx.double(), x64.grad, rtol=0, atol=20 * 2.0 ** -24 * g.abs().max().item())
    step = torch.zeros_like(x)                              # the map is linear: a difference of any size is the slope
    step[4, 1, 3] = 1024.0
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    rope(cass, x, None, y0, None, freqs, pos, rot, interleaved)
    rope(cass, x + step, None, y1, None, freqs, pos, rot, interleaved)
    slope = ((y1.double() - y0.double()) * g.double()).sum().item() / 1024.0
    assert abs(slope - gx[4, 1, 3].item()) <= 64 * 2.0 ** -24 * 1040 / 1024 * g.abs().max().item()


def test_streams_and_graphs(cass):
    rows, n, d = 50, 4, 64
    freqs = device_freqs(cass, d, "none")
    x = torch.randn(rows, n, d, device="cuda").to(torch.bfloat16)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    want, got = torch.empty_like(x), torch.zeros_like(x)
    rope(cass, x, None, want, None, freqs, pos, d, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rope(cass, x, None, got, None, freqs, pos, d, False, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rope(cass, x, None, got, None, freqs, pos, d, False)
    x.copy_(torch.randn(rows, n, d, device="cuda"))
    pos.add_(1000)
    graph.replay()
    rope(cass, x, None, want, None, freqs, pos, d, False)
    assert torch.equal(got, want)


def test_session_with_scaled_positions(cass):
    """Unscaled parameters leave a session's results alone, bit for bit; scaled by 2, every second position is turned as the positions of
    the unscaled session are; what does not fit the head is refused."""
    import dataclasses

    import synth
    from paper_2605_26558_b200 import engine
    shape = dataclasses.replace(synth.TINY, n_layers=1)
    w = synth.model_weights(shape, 5, "cuda")
    w["layers"] = [engine.fuse_layer_weights(lw) for lw in w["layers"]]
    eng = engine.Engine(shape, w, max_seq=128)
    toks = torch.full((1, 5), 77, device="cuda", dtype=torch.int32)          # one token everywhere: rows differ by their positions alone

    def rows():
        out = torch.zeros(5, shape.vocab, device="cuda")
        eng.reset()
        cass.cass_verify(eng.session, toks, 4, torch.zeros(5, dtype=torch.int32, device="cuda"), out)
        ptr, _, cols = cass.cass_debug_activation(eng.session, 2)
        o = ptr - eng.mem.data_ptr()
        return out, eng.mem[o: o + 2 * 5 * cols].view(torch.bfloat16).view(5, cols).clone()

    logits, turned = rows()
    params = lambda kind, s=2.0: cass.RopeParams(shape.head_dim, kind, shape.rope_theta, s, 1.0, 4.0, 64.0, 0.0)  # noqa: E731
    cass.cass_session_set_rope(eng.session, params(cass.ROPE_PLAIN))
    same, same_turned = rows()
    assert torch.equal(logits, same) and torch.equal(turned, same_turned)
    cass.cass_session_set_rope(eng.session, params(cass.ROPE_LINEAR))
    _, scaled_turned = rows()                               # (one token's values are the same everywhere, and so are the logits)
    assert torch.equal(scaled_turned[::2], turned[:3]) and not torch.equal(scaled_turned[1], turned[1])
    with pytest.raises(cass.CassError) as e:
        cass.cass_session_set_rope(eng.session, cass.RopeParams(32, 0, 1e4, 1.0, 1.0, 4.0, 64.0, 0.0))
    assert e.value.code == cass.ERR_UNSUPPORTED
    with pytest.raises(cass.CassError):
        cass.cass_session_set_rope(eng.session, params(cass.ROPE_LINEAR, -1.0))
    eng.close()
