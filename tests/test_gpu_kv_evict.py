"""Eviction (cass_kv_evict) against a plain selection: which positions stay, that their rows and weights move unchanged, and what is left alone."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


def cache(cass, t):
    """[sequence][position][head][dim], any order in memory."""
    kind = {torch.bfloat16: cass.BF16, torch.float16: cass.F16}[t.dtype]
    return cass.CacheGeom(kind, t.shape[0], t.shape[2], t.shape[3], t.shape[1], t.stride(0), t.stride(1), t.stride(2))


def order(t, how):
    return t if how == "bphd" else t.transpose(1, 2).contiguous().transpose(1, 2) if how == "bhpd" else t.transpose(0, 1).contiguous().transpose(0, 1)


def stays(w, n, budget, first, last):
    """Positions that stay, by the definition."""
    if n <= budget:
        return list(range(n))
    key = lambda j: -math.inf if math.isnan(w[j]) else w[j]  # noqa: E731
    nan = lambda j: math.isnan(w[j])  # noqa: E731
    mid = sorted(range(first, n - last), key=lambda j: (nan(j), -key(j), j))[: budget - first - last]
    return sorted(list(range(first)) + mid + list(range(n - last, n)))


def run(cass, k, v, w, lens, budget, first, last, out=None, w_out=True, alias=False):
    b, cap, h, _ = k.shape
    kept = torch.full((b, h, budget), -7, dtype=torch.int32, device="cuda")
    new = lens if alias else torch.full_like(lens, -9)
    if out is None:
        wo = w if w_out else None
        cass.cass_kv_evict(cache(cass, k), k.data_ptr(), v.data_ptr(), w, lens, budget, first, last, None, None, None, wo, kept, new)
    else:
        wo = torch.full((b, h, out[0].shape[1]), -3.0, device="cuda") if w_out else None
        cass.cass_kv_evict(cache(cass, k), k.data_ptr(), v.data_ptr(), w, lens, budget, first, last, cache(cass, out[0]), out[0].data_ptr(),
                           out[1].data_ptr(), wo, kept, new)
    return kept, new, wo


def bits(t):
    return t.contiguous().view(torch.int16) if t.element_size() == 2 else t.contiguous().view(torch.int32)


def check(cass, k, v, w, lens, budget, first, last, out_cap=None, how="bphd", w_out=True, alias=False):
    b, cap, h, d = k.shape
    k0, v0, w0, l0 = k.clone(), v.clone(), w.clone(), lens.tolist()
    out = None
    if out_cap is not None:
        out = tuple(order(torch.full((b, out_cap, h, d), 3.0, dtype=k.dtype, device="cuda"), how) for _ in range(2))
    kept, new, wo = run(cass, k, v, w, lens, budget, first, last, out, w_out, alias)
    ko, vo = (k, v) if out is None else out
    before = (k0, v0) if out is None else tuple(torch.full_like(x, 3.0) for x in out)
    ws = w0.cpu().tolist()
    for i in range(b):
        n = l0[i]
        there = 0 <= n <= cap
        assert int(new[i]) == (min(n, budget) if there else n)
        for j in range(h):
            want = stays(ws[i][j], n, budget, first, last) if there else []
            got = kept[i, j].tolist()
            assert got == want + [-1] * (budget - len(want)), (i, j, n)
            at, m = torch.tensor(want, dtype=torch.long, device="cuda"), len(want)
            for x, y, z in ((ko, k0, before[0]), (vo, v0, before[1])):
                assert torch.equal(bits(x[i, :m, j]), bits(y[i, at, j]))
                assert torch.equal(bits(x[i, m:, j]), bits(z[i, m:, j]))
            if wo is not None and there:
                assert torch.equal(bits(wo[i, j, :m]), bits(w0[i, j, at])) and (wo[i, j, m:] == 0).all()
            elif wo is not None:
                assert torch.equal(bits(wo[i, j]), bits(w0[i, j])) if out is None else (wo[i, j] == -3.0).all()
    if out is not None:
        assert torch.equal(bits(k), bits(k0)) and torch.equal(bits(v), bits(v0)) and torch.equal(bits(w), bits(w0))


def make(b, cap, h, d, dtype=torch.bfloat16, how="bphd", seed=0, ties=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (order(torch.randn(b, cap, h, d, generator=g, device="cuda").to(dtype), how) for _ in range(2))
    w = torch.exp(torch.randn(b, h, cap, generator=g, device="cuda") * 2)
    if ties:
        w = torch.where(w < 0.7, torch.zeros_like(w), (w * 8).round() / 8)
    return k, v, w


@pytest.mark.parametrize("how", ["bphd", "bhpd", "pbhd"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("b,cap,h,d,budget,first,last", [
    (1, 40, 2, 64, 16, 2, 4), (3, 257, 2, 128, 100, 0, 0), (2, 1000, 3, 96, 999, 4, 16), (2, 1000, 1, 8, 1, 0, 0), (1, 1, 1, 64, 1, 0, 0),
    (2, 700, 2, 128, 64, 32, 32), (2, 700, 2, 128, 64, 64, 0), (2, 700, 2, 128, 64, 0, 64), (1, 9000, 8, 128, 4096, 16, 512), (5, 33, 1, 512, 20, 1, 1),
    (4, 128, 2, 24, 128, 3, 9)])
def test_out_of_place_and_in_place(cass, how, dtype, b, cap, h, d, budget, first, last):
    for ragged in (False, True):
        k, v, w = make(b, cap, h, d, dtype, how, cap + budget)
        g = torch.Generator().manual_seed(cap)
        lens = torch.randint(0, cap + 1, (b,), generator=g, dtype=torch.int32).cuda() if ragged else torch.full((b,), cap, dtype=torch.int32, device="cuda")
        check(cass, k, v, w, lens.clone(), budget, first, last, out_cap=budget, how=how)
        check(cass, k, v, w, lens.clone(), budget, first, last, out_cap=budget + 5, how="bhpd", w_out=False)
        check(cass, k, v, w, lens.clone(), budget, first, last)
        k, v, w = make(b, cap, h, d, dtype, how, cap)
        check(cass, k, v, w, lens.clone(), budget, first, last, w_out=False, alias=True)


@pytest.mark.parametrize("cap,h", [(20000, 1), (33000, 4), (100003, 2), (400000, 1)])
def test_long_caches(cass, cap, h):
    """Several CTAs a head, and more positions than they keep in shared memory."""
    k, v, w = make(1, cap, h, 8, seed=cap)
    lens = torch.tensor([cap - 3], dtype=torch.int32, device="cuda")
    check(cass, k, v, w, lens.clone(), cap // 3, 5, 1000, out_cap=cap // 3)
    check(cass, k, v, w, lens, cap - 1000, 5, 1000, alias=True)


def test_weights_that_are_hard_to_order(cass):
    inf, nan = math.inf, math.nan
    rows = [[0.0] * 50, [-0.0, 0.0] * 25, [nan] * 50, [inf] * 25 + [nan] * 25, [-inf] * 10 + [nan] * 30 + [-1.0] * 10, [1e-45, -1e-45, 0.0, -0.0, 1e-38] * 10,
            list(range(50)), list(range(50, 0, -1)), [3.0] * 20 + [nan, inf, -inf, 0.0, -0.0] * 6, [3.4028234e38, -3.4028234e38] * 25]
    w = torch.tensor(rows, device="cuda").view(5, 2, 50)
    lens = torch.tensor([50, 50, 49, 30, 50], dtype=torch.int32, device="cuda")
    for budget, first, last in ((20, 0, 0), (20, 3, 5), (1, 0, 0), (49, 0, 0), (20, 10, 10)):
        k, v, _ = make(5, 50, 2, 16, seed=budget)
        check(cass, k, v, w.clone(), lens.clone(), budget, first, last, out_cap=budget)
        check(cass, k, v, w.clone(), lens.clone(), budget, first, last)


def test_zeros_right_behind_the_largest_weights(cass):
    """Negative weights down to the smallest number and some zeros: the zeros stay, and so do the weights next to them."""
    for cap, near, zeros in ((500, 7, 3), (3000, 60, 40), (9000, 300, 5), (20000, 2, 1)):
        k, v, w = make(1, cap, 2, 64, seed=cap)
        w = -(1 + w)
        g = torch.Generator(device="cuda").manual_seed(cap)
        at = torch.randperm(cap, generator=g, device="cuda")
        w[:, :, at[:near]] = -torch.arange(1, near + 1, device="cuda", dtype=torch.int32).view(torch.float32)       # steps of 2^-149
        w[:, :, at[near: near + zeros]] = 0.0
        for budget in (1, zeros, zeros + 1, zeros + near - 1, zeros + near, zeros + near + 5):
            check(cass, k.clone(), v.clone(), w.clone(), torch.tensor([cap], dtype=torch.int32, device="cuda"), budget, 0, 0)


def test_a_budget_beyond_the_first_cache(cass):
    """Into a larger cache: everything stays."""
    k, v, w = make(3, 60, 2, 64)
    check(cass, k, v, w, torch.tensor([60, 0, 59], dtype=torch.int32, device="cuda"), 80, 2, 4, out_cap=90)


def test_lengths_that_mean_nothing_leave_a_sequence_alone(cass):
    k, v, w = make(5, 60, 2, 64)
    lens = torch.tensor([61, -1, 60, 0, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    check(cass, k, v, w, lens.clone(), 30, 2, 4, out_cap=32)
    check(cass, k, v, w, lens.clone(), 30, 2, 4, alias=True)


def test_values_that_are_no_numbers_move_as_they_are(cass):
    k, v, w = make(2, 300, 2, 128)
    k.view(torch.int16).random_(-32768, 32767)
    v.view(torch.int16).random_(-32768, 32767)
    lens = torch.tensor([300, 299], dtype=torch.int32, device="cuda")
    check(cass, k, v, w, lens, 77, 1, 10)


def test_graph_and_repeated_eviction(cass):
    """A captured in-place eviction, replayed as the cache fills again: each time as a fresh call would do it."""
    k, v, w = make(2, 200, 2, 64, seed=3)
    lens = torch.tensor([200, 150], dtype=torch.int32, device="cuda")
    kept = torch.zeros(2, 2, 120, dtype=torch.int32, device="cuda")
    g = cache(cass, k)
    state = [x.clone() for x in (k, v, w, lens)]
    call = lambda k, v, w, lens: cass.cass_kv_evict(g, k.data_ptr(), v.data_ptr(), w, lens, 120, 4, 16, None, None, None, w, kept, lens)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(*[x.clone() for x in state])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(k, v, w, lens)
    for step in range(3):
        graph.replay()
        call(*state)
        assert all(torch.equal(x, y) for x, y in zip((k, v, w, lens), state))
        assert lens.tolist() == [120, 120]
        for x, y in zip((k, v, w, lens), state):            # the caches fill again
            fill = torch.randn(2, 60, 2, 64, device="cuda").to(k.dtype)
            if x.dim() == 4:
                x[:, 120:180], y[:, 120:180] = fill, fill
            elif x.dim() == 3:
                x[..., 120:180] = y[..., 120:180] = torch.rand(2, 2, 60, device="cuda")
            else:
                x.fill_(180), y.fill_(180)


def test_offsets_beyond_32_bits(cass):
    """The second sequence lies more than 2^32 bytes behind the first."""
    far = (1 << 31) + (1 << 20)                             # elements
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("no room for a cache of that size")
    flat = torch.empty(far + 200 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    k = flat.as_strided((2, 200, 2, 64), (far, 128, 64, 1))
    k.copy_(torch.randn(2, 200, 2, 64, device="cuda"))
    v = k.clone()
    w = torch.rand(2, 2, 200, device="cuda")
    k0 = k.clone()
    lens = torch.tensor([200, 180], dtype=torch.int32, device="cuda")
    kept = torch.zeros(2, 2, 50, dtype=torch.int32, device="cuda")
    vg = v.as_strided((2, 200, 2, 64), (200 * 128, 128, 64, 1))
    out = cass.CacheGeom(cass.BF16, 2, 2, 64, 50, 50 * 128, 128, 64)
    ko, vo = (torch.zeros(2, 50, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    big_v = torch.empty_like(flat)
    big_v.as_strided((2, 200, 2, 64), (far, 128, 64, 1)).copy_(vg)
    cass.cass_kv_evict(cache(cass, k), k.data_ptr(), big_v.data_ptr(), w, lens, 50, 2, 3, out, ko.data_ptr(), vo.data_ptr(), None, kept, lens)
    for i, n in enumerate((200, 180)):
        for j in range(2):
            want = stays(w[i, j].tolist(), n, 50, 2, 3)
            assert kept[i, j].tolist() == want
            assert torch.equal(ko[i, :, j], k0[i, want, j]) and torch.equal(vo[i, :, j], k0[i, want, j])
