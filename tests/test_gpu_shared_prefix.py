"""Attention behind a shared prefix (cass_shared_prefix_attention) against the definition in 64 bits.

Tolerances.  Scores: exact products of 16-bit values, summed in 32 bits by the matrix units in d / 16 steps (taken as 2^-23 of the sum
of their absolute values a step, truncation included) and scaled (2^-24 twice): ds = scale sum|q k| (d / 16 + 2) 2^-23.  A probability is
then off by a factor of 1 + 2 ds + 2^-21 (the exponential, and the scores' rescaling to powers of two: 2^-24 |s| of 1.45 |s|, with
|s| <= 64).  Sums of n of them in 32 bits: chains of at most n / 16 + 64 additions, 2^-24 each.  The second product takes probabilities
rounded to the type (eps / 2 each) and adds 2^-23 a step of 16 positions.  Outputs add half a step of their type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


def kind(cass, t):
    return {torch.bfloat16: cass.BF16, torch.float16: cass.F16}[t.dtype]


class Case:
    """Inputs of one call; sequences with a length below 0 are not there."""

    def __init__(self, b, rows, nq, nk, d, prefix, cap, lens, dtype=torch.bfloat16, how="bphd", seed=0, scale=0.0, garbage=True):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *n: torch.randn(*n, generator=g, device="cuda").to(dtype)  # noqa: E731
        order = lambda t: t if how == "bphd" else t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
        self.b, self.rows, self.nq, self.nk, self.d, self.prefix, self.cap, self.lens, self.scale = b, rows, nq, nk, d, prefix, cap, list(lens), scale
        self.q = rnd(b, rows, nq, d)
        self.kp, self.vp = order(rnd(1, prefix, nk, d))[0], order(rnd(1, prefix, nk, d))[0]
        self.kc, self.vc = order(rnd(b, cap, nk, d)), order(rnd(b, cap, nk, d))
        if garbage:                                         # what no row sees may be anything
            for i, n in enumerate(self.lens):
                n = min(max(n, 0), cap)
                self.kc[i, n:], self.vc[i, n:] = math.nan, math.inf
        self.w_in = torch.rand(b, nk, cap, generator=g, device="cuda")

    def geoms(self, cass):
        c, p = self.kc, self.kp
        st = self.q.stride()
        cg = cass.CacheGeom(kind(cass, self.q), self.b, self.nk, self.d, self.cap, c.stride(0), c.stride(1), c.stride(2))
        return cg, cass.SharedAttn(self.nq, self.rows, st[0], st[1], st[2], *self.out_strides(), self.prefix, p.stride(0), p.stride(1), self.scale)

    def out_strides(self):
        return self.rows * self.nq * self.d, self.nq * self.d, self.d

    def run(self, cass, weights=True, scratch=None, stream=None, in_place=False):
        cg, ag = self.geoms(cass)
        out = torch.full((self.b, self.rows, self.nq, self.d), 9.0, dtype=self.q.dtype, device="cuda")
        lse = torch.full((self.b, self.rows, self.nq), 9.0, device="cuda")
        w_in = self.w_in.clone() if in_place else self.w_in
        w = (w_in if in_place else torch.full_like(self.w_in, 9.0)) if weights else None
        lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        need = cass.cass_shared_prefix_scratch_bytes(cg, ag, weights)
        if scratch is None:
            scratch = torch.full((need + 64,), 0x7F, dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cass.cass_shared_prefix_attention(cg, ag, self.q, self.kp.data_ptr() if self.prefix else None, self.vp.data_ptr() if self.prefix else None,
                                          self.kc.data_ptr() if self.cap else None, self.vc.data_ptr() if self.cap else None, lens if self.cap else None,
                                          out, lse, w_in if weights else None, w, scratch, need, status, stream)
        if scratch.numel() == need + 64:
            torch.cuda.synchronize()
            assert (scratch[need:] == 0x7F).all()           # nothing behind the scratch
        return out, lse, w, status

    def check(self, cass, weights=True, **kw):
        out, lse, w, status = self.run(cass, weights, **kw)
        clipped = any(n > self.cap for n in self.lens)
        assert int(status.item()) == (cass.ERR_CAPACITY if clipped else 0)
        scale = self.scale or self.d ** -0.5
        grp, half = self.nq // self.nk, torch.finfo(self.q.dtype).eps / 2
        for b, n in enumerate(self.lens):
            if n < 0:
                assert (out[b] == 9.0).all() and (lse[b] == 9.0).all() and (w is None or (w[b] == 9.0).all() or torch.equal(w[b], self.w_in[b]))
                continue
            n = min(n, self.cap)
            for h in range(self.nk):
                hs = slice(h * grp, (h + 1) * grp)
                k, v = torch.cat((self.kp[:, h], self.kc[b, :n, h])).double(), torch.cat((self.vp[:, h], self.vc[b, :n, h])).double()
                total, total_tol = self.w_in[b, h].double().clone(), torch.zeros(self.cap, dtype=torch.float64, device="cuda")
                for r in range(self.rows):
                    end = self.prefix + max(n - (self.rows - 1 - r), 0)
                    if end == 0:
                        assert (out[b, r, hs] == 0).all() and (lse[b, r, hs] == -math.inf).all()
                        continue
                    q = self.q[b, r, hs].double()
                    s = q @ k[:end].T * scale
                    ds = (q.abs() @ k[:end].abs().T).amax(1, keepdim=True) * scale * (self.d / 16 + 2) * 2.0 ** -23
                    z = torch.logsumexp(s, 1, keepdim=True)
                    p = torch.exp(s - z)
                    rel = 2 * ds + 2.0 ** -21 + s.abs().amax(1, keepdim=True).clamp(min=1) * 2.0 ** -23
                    chain = (end / 16 + 64) * 2.0 ** -24
                    o, size = p @ v[:end], p @ v[:end].abs()
                    tol = size * (half + 2 * rel + chain + (end / 16 + 16) * 2.0 ** -23) + o.abs() * half * 1.01 + 2.0 ** -25
                    err = (out[b, r, hs].double() - o).abs()
                    assert (err <= tol).all(), ("out", b, h, r, (err / tol).max().item())
                    err = (lse[b, r, hs].double() - z[:, 0]).abs()
                    assert (err <= (ds + 2.0 ** -20 + chain)[:, 0] + z[:, 0].abs() * 2.0 ** -22).all(), ("lse", b, h, r, err.max().item())
                    total[: end - self.prefix] += p[:, self.prefix:].sum(0)
                    total_tol[: end - self.prefix] += (p[:, self.prefix:] * (2 * rel + chain)).sum(0)
                if w is not None:
                    err = (w[b, h].double() - total).abs()
                    assert (err <= total_tol + total.abs() * (self.rows * grp + 2) * 2.0 ** -24).all(), ("weights", b, h, err.max().item())
        return out, lse, w


HEADS = [(4, 2, 64), (32, 8, 128), (40, 8, 128), (5, 5, 32), (16, 1, 96), (6, 2, 192), (8, 2, 256), (7, 1, 64)]


@pytest.mark.parametrize("nq,nk,d", HEADS)
@pytest.mark.parametrize("dtype,how", [(torch.bfloat16, "bphd"), (torch.float16, "bhpd")])
@pytest.mark.parametrize("b,rows,prefix,cap,lens", [
    (1, 1, 0, 1, [1]), (1, 1, 0, 1, [0]), (1, 1, 1, 0, [0]), (2, 1, 100, 33, [1, 33]), (3, 5, 63, 70, [5, 64, 70]), (3, 3, 64, 130, [0, 1, 129]),
    (2, 16, 65, 65, [16, 65]), (4, 2, 129, 300, [-1, 2, 299, 257]), (5, 1, 1000, 64, [0, 64, 1, -3, 63])])
def test_against_the_definition(cass, nq, nk, d, dtype, how, b, rows, prefix, cap, lens):
    Case(b, rows, nq, nk, d, prefix, cap, lens, dtype, how, seed=prefix + cap).check(cass, weights=cap > 0)


@pytest.mark.parametrize("nq,nk,d", [(4, 2, 64), (32, 8, 128), (24, 2, 128), (4, 2, 32), (2, 1, 256)])
@pytest.mark.parametrize("b,rows,prefix", [(9, 1, 700), (20, 1, 130), (33, 2, 257), (64, 1, 128), (70, 3, 500), (16, 16, 200), (150, 1, 90)])
def test_many_sequences_behind_a_prefix(cass, nq, nk, d, b, rows, prefix):
    lens = [(37 * i) % 90 + (0 if i % 7 else -90) for i in range(b)]
    Case(b, rows, nq, nk, d, prefix, 90, lens, torch.bfloat16 if b % 2 else torch.float16, seed=b).check(cass, weights=b % 3 == 0)


def test_long_caches_and_prefixes(cass):
    Case(1, 1, 32, 8, 128, 0, 30000, [29999], how="bhpd").check(cass)
    Case(2, 5, 4, 2, 64, 9001, 5000, [5000, 3], torch.float16).check(cass)
    Case(40, 1, 8, 2, 128, 8191, 10, [7] * 40).check(cass, weights=False)
    Case(3, 1, 8, 1, 256, 4000, 2000, [1, 2000, 600]).check(cass)


@pytest.mark.parametrize("nq,nk,d,b,rows", [(8, 2, 128, 2, 1), (8, 2, 128, 40, 1), (4, 2, 64, 2, 4), (4, 2, 64, 70, 1), (4, 2, 96, 3, 2)])
def test_large_scores(cass, nq, nk, d, b, rows):
    """Maxima that grow along the positions, by far more than the exponential's range: what came before has to vanish, not overflow."""
    c = Case(b, rows, nq, nk, d, 500, 200, [200] * b, scale=0.05)
    c.kp *= torch.linspace(0.1, 6, 500, device="cuda")[:, None, None].to(c.kp.dtype)
    c.kc *= torch.linspace(6, 9, 200, device="cuda")[None, :, None, None].to(c.kc.dtype)
    c.check(cass)
    c.q *= 0
    c.check(cass)                                           # all alike


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_a_row_does_not_see_does_not_reach_it(cass, dtype, d):
    """The keys and values of later rows hold no numbers: rows before them are as if those were zeros; rows that see them follow the formula."""
    for bad_k, bad_v in ((0.5, math.nan), (math.nan, 1.0), (0.5, math.inf), (math.nan, math.nan), (-math.inf, math.nan)):
        c = Case(3, 5, 8, 2, d, 70, 150, [140, 64, 5], dtype, seed=d)
        clean = Case(3, 5, 8, 2, d, 70, 150, [140, 64, 5], dtype, seed=d)
        for i, n in enumerate(c.lens):
            c.kc[i, n - 2:n, :, ::3], c.vc[i, n - 2:n, 1, 1::5] = bad_k, bad_v
            clean.kc[i, n - 2:n], clean.vc[i, n - 2:n] = 0, 0
        out, lse, _, _ = c.run(cass)
        want, want_lse, _, _ = clean.run(cass)
        assert torch.equal(out[:, :3], want[:, :3]) and torch.equal(lse[:, :3], want_lse[:, :3])
        if math.isnan(bad_k):
            assert out[:, 3:].isnan().all()
        elif bad_k == 0.5:
            seen = torch.zeros(d, dtype=torch.bool, device="cuda")
            seen[1::5] = True
            for r in (3, 4):
                assert (out[:, r, 4:][..., seen].isnan() if math.isnan(bad_v) else out[:, r, 4:][..., seen] == math.inf).all()
                assert out[:, r, 4:][..., ~seen].isfinite().all() and out[:, r, :4].isfinite().all()


@pytest.mark.parametrize("b", [2, 60])
def test_infinite_scores(cass, b):
    """A key at the type's infinity for one pair: its row follows the formula (no number), the others are as without it."""
    c, clean = (Case(b, 1, 8, 2, 128, 300, 50, [40] * b) for _ in range(2))
    c.kp[150, 0, 0] = math.inf
    out, _, _, _ = c.run(cass)
    want, _, _, _ = clean.run(cass)
    assert torch.equal(out[:, :, 4:], want[:, :, 4:])
    neg = c.q[:, 0, :4, 0] < 0                              # a score of -inf: the position has no weight
    assert out[:, 0, :4][neg].isfinite().all() and out[:, 0, :4][~neg].isnan().all()


def test_nothing_to_see(cass):
    """No prefix and no cache: outputs 0, log sums -inf."""
    c = Case(3, 2, 8, 2, 64, 0, 0, [0, 0, 0])
    out, lse, _, status = c.run(cass, weights=False)
    assert (out == 0).all() and (lse == -math.inf).all() and int(status.item()) == 0


@pytest.mark.parametrize("nq,nk,d,rows,cap", [(40, 8, 128, 5, 700), (16, 1, 64, 16, 300), (32, 2, 128, 3, 200), (12, 4, 256, 7, 150)])
def test_many_rows_of_a_sequence(cass, nq, nk, d, rows, cap):
    """More pairs of a sequence and head than one, two or four tiles of 16 hold."""
    Case(3, rows, nq, nk, d, 130, cap, [cap, rows, cap // 2], torch.float16, seed=rows).check(cass)


@pytest.mark.parametrize("d", [64, 128, 96])
@pytest.mark.parametrize("nq,nk,rows", [(16, 2, 5), (16, 1, 4), (4, 2, 2)])
def test_values_that_are_no_numbers_behind_several_tiles_of_pairs(cass, d, nq, nk, rows):
    c, clean = (Case(2, rows, nq, nk, d, 40, 200, [200, 67], seed=d) for _ in range(2))
    for i, n in enumerate(c.lens):
        c.vc[i, n - 1, :, 3::7], clean.vc[i, n - 1] = math.nan, 0
    out, lse, _, _ = c.run(cass)
    want, want_lse, _, _ = clean.run(cass)
    assert torch.equal(out[:, :-1], want[:, :-1]) and torch.equal(lse, want_lse)
    bad = torch.zeros(d, dtype=torch.bool, device="cuda")
    bad[3::7] = True
    assert out[:, -1][..., bad].isnan().all() and out[:, -1][..., ~bad].isfinite().all()


def test_lengths_beyond_the_capacity_are_cut(cass):
    Case(3, 2, 8, 2, 64, 20, 50, [51, 50, 2 ** 31 - 1]).check(cass)


def test_weights_in_place_without_and_repeated(cass):
    c = Case(4, 3, 8, 2, 128, 100, 600, [600, 3, 0, 333])
    out, lse, w = c.check(cass)
    out2, lse2, w2, _ = c.run(cass, in_place=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(w, w2)
    out3, lse3, _, _ = c.run(cass, weights=False)
    assert torch.equal(out, out3) and torch.equal(lse, lse3)
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(c.run(cass)[:3], (out, lse, w)))


def test_strided_queries_and_outputs(cass):
    """q inside packed rows, the output heads before rows; what lies between is left alone."""
    c = Case(3, 2, 8, 2, 64, 90, 70, [70, 2, 33])
    want, lse, _, _ = c.run(cass)
    packed = torch.randn(3, 2, 12, 64, device="cuda").to(torch.bfloat16)
    packed[:, :, :8] = c.q
    out = torch.full((3, 8, 2, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    cg, ag = c.geoms(cass)
    ag.q_seq, ag.q_row, ag.q_head = packed.stride()[:3]
    ag.out_seq, ag.out_row, ag.out_head = out.stride(0), out.stride(2), out.stride(1)
    scratch = torch.zeros(cass.cass_shared_prefix_scratch_bytes(cg, ag), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    cass.cass_shared_prefix_attention(cg, ag, packed, c.kp, c.vp, c.kc, c.vc, lens, out, None, None, None, scratch, scratch.numel(), status)
    assert torch.equal(out[..., :64].transpose(1, 2), want) and (out[..., 64:] == 5.0).all()


def test_streams_graphs_and_new_lengths(cass):
    """A captured call follows the lengths that the device holds when it is replayed; its scratch may hold anything."""
    c = Case(4, 1, 8, 2, 128, 300, 400, [400] * 4, garbage=False)
    cg, ag = c.geoms(cass)
    lens = torch.tensor([10, 20, 30, 40], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(c.q), torch.zeros(4, 1, 8, device="cuda")
    scratch = torch.zeros(cass.cass_shared_prefix_scratch_bytes(cg, ag), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda s=None: cass.cass_shared_prefix_attention(cg, ag, c.q, c.kp, c.vp, c.kc, c.vc, lens, out, lse, None, None, scratch,  # noqa: E731
                                                            scratch.numel(), status, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new in ([400, 1, 0, 77], [-1, 400, 399, 64]):
        lens.copy_(torch.tensor(new))
        scratch.fill_(0xFF)
        out.fill_(9.0)
        lse.fill_(9.0)
        graph.replay()
        c.lens = new
        want, want_lse, _, _ = c.run(cass, weights=False)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_two_calls_at_once(cass):
    """Two streams with scratch of their own, over and over: each gets its own results."""
    cases = [Case(3, 1, 8, 2, 128, 2000, 500, [500, 3, 77], seed=1), Case(40, 2, 8, 2, 128, 900, 100, [50] * 40, seed=2)]
    want = [c.run(cass)[:3] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(c.run(cass, scratch=torch.empty(cass.cass_shared_prefix_scratch_bytes(*c.geoms(cass), True), dtype=torch.uint8, device="cuda"))[:3])
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_offsets_beyond_32_bits(cass):
    """The second sequence's cache, and the last of a prefix, more than 2^32 bytes behind the first."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("no room for a cache of that size")
    far = (1 << 31) + 1024
    c = Case(2, 2, 4, 2, 64, 100, 80, [80, 77])
    want = c.run(cass)[:3]
    big = []
    for t in (c.kc, c.vc):
        flat = torch.empty(far + 80 * 128, dtype=t.dtype, device="cuda")
        v = flat.as_strided((2, 80, 2, 64), (far, 128, 64, 1))
        v.copy_(t)
        big.append(v)
    c.kc, c.vc = big
    got = c.run(cass)[:3]
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    c.kc, c.vc = (t.contiguous() for t in big)
    del big, v, flat
    step = 22 << 20                                         # elements between a prefix's positions: the last ones beyond 2^31
    flats = [torch.empty(99 * step + 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = [f.as_strided((100, 2, 64), (step, 64, 1)) for f in flats]
    views[0].copy_(c.kp)
    views[1].copy_(c.vp)
    c.kp, c.vp = views
    got = c.run(cass)[:3]
    assert all(torch.equal(x, y) for x, y in zip(got, want))
