"""Eviction from a cache of the largest capacity (its positions are as many as its length says)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


@pytest.mark.parametrize("capacity", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30])
@pytest.mark.parametrize("n,budget", [(20000, 5000), (150000, 70001), (3000, 3000), (100, 3000)])
def test_the_largest_capacity(cass, capacity, n, budget):
    """Nothing behind a sequence's length is read or written, so the buffers need not hold the capacity."""
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn(n, 8, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randn(n, generator=g, device="cuda")
    first, last = 3, 100
    stay = torch.arange(n, device="cuda")
    if n > budget:
        best = torch.sort(w[first: n - last], descending=True, stable=True).indices[: budget - first - last] + first
        stay = torch.cat((stay[:first], best.sort().values, stay[n - last:]))
    want_k, want_v = k[stay], v[stay]
    lens, kept = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(budget, dtype=torch.int32, device="cuda")
    geom = cass.CacheGeom(cass.BF16, 1, 1, 8, capacity, 0, 8, 0)
    cass.cass_kv_evict(geom, k, v, w, lens, budget, first, last, None, None, None, None, kept, lens)
    assert kept[: len(stay)].tolist() == stay.tolist() and (kept[len(stay):] == -1).all()
    assert int(lens.item()) == len(stay) and torch.equal(k[: len(stay)], want_k) and torch.equal(v[: len(stay)], want_v)
