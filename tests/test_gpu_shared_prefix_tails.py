"""Attention whose scores are one or a few large ones before a long tail of small ones, as trained models have them: the tail's share
of the output is small a position and large together.

Tolerances are those of test_gpu_shared_prefix.py, and one term more: a numerator below the type's smallest normal number is off by half
a step of its subnormal ones.  fp16 numerators are kept relative to 2^11 or more, so that is 2^-25 / 2^11 of the largest, n of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("b,rows,nq,nk,d,prefix,cap", [
    (1, 1, 8, 2, 128, 0, 32768), (2, 5, 8, 1, 64, 0, 9000), (2, 1, 4, 1, 128, 32768, 40), (2, 1, 8, 2, 256, 20000, 40), (24, 1, 8, 2, 96, 9000, 10),
    (16, 1, 32, 8, 128, 32768, 20), (40, 1, 4, 1, 64, 32768, 20), (64, 2, 8, 2, 128, 32768, 20), (70, 3, 8, 2, 64, 16000, 20)])
def test_a_long_tail_behind_favoured_positions(cass, dtype, b, rows, nq, nk, d, prefix, cap):
    """Every thousandth position scores 17 more than the others and has a value of 0: what comes out is the tail's."""
    g = torch.Generator(device="cuda").manual_seed(prefix + cap)
    rnd = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    q = rnd(b, rows, nq, d) * 0.05
    q[..., 0] = 4.0
    keys, values = [], []
    for n in (prefix, b * cap):
        k, v = rnd(n, nk, d), 64 + 8 * rnd(n, nk, d)
        k[:, :, 0] = 0
        favoured = torch.arange(n, device="cuda") % 1000 == 0
        k[favoured, :, 0], v[favoured] = 17 / 4, 0
        keys.append(k.to(dtype))
        values.append(v.to(dtype))
    q, (kp, kc), (vp, vc) = q.to(dtype), keys, values
    kc, vc = kc.view(b, cap, nk, d), vc.view(b, cap, nk, d)
    kind = cass.BF16 if dtype == torch.bfloat16 else cass.F16
    geom = cass.CacheGeom(kind, b, nk, d, cap, *kc.stride()[:3])
    attn = cass.SharedAttn(nq, rows, *q.stride()[:3], *q.stride()[:3], prefix, nk * d, d, 1.0)
    scratch = torch.zeros(cass.cass_shared_prefix_scratch_bytes(geom, attn, True), dtype=torch.uint8, device="cuda")
    status, lens = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((b,), cap, dtype=torch.int32, device="cuda")
    out, lse, w = torch.zeros_like(q), torch.zeros(b, rows, nq, device="cuda"), torch.zeros(b, nk, cap, device="cuda")
    cass.cass_shared_prefix_attention(geom, attn, q, kp if prefix else None, vp if prefix else None, kc, vc, lens, out, lse, None, w, scratch,
                                      scratch.numel(), status)
    assert int(status.item()) == 0
    grp, half = nq // nk, torch.finfo(dtype).eps / 2
    for i in sorted({0, b // 2, b - 1}):
        for h in range(nk):
            k, v = torch.cat((kp[:, h], kc[i, :, h])).double(), torch.cat((vp[:, h], vc[i, :, h])).double()
            total, total_tol = torch.zeros(cap, dtype=torch.float64, device="cuda"), torch.zeros(cap, dtype=torch.float64, device="cuda")
            for r in range(rows):
                end, hs = prefix + cap - (rows - 1 - r), slice(h * grp, (h + 1) * grp)
                x = q[i, r, hs].double()
                s = x @ k[:end].T
                ds = (x.abs() @ k[:end].abs().T).amax(1, keepdim=True) * (d / 16 + 2) * 2.0 ** -23
                z = torch.logsumexp(s, 1, keepdim=True)
                p = torch.exp(s - z)
                rel = 2 * ds + 2.0 ** -21 + s.abs().amax(1, keepdim=True).clamp(min=1) * 2.0 ** -23
                chain = (end / 16 + 64) * 2.0 ** -24
                o, size = p @ v[:end], p @ v[:end].abs()
                tol = size * (half + 2 * rel + chain + (end / 16 + 16) * 2.0 ** -23) + o.abs() * half * 1.01 + 2.0 ** -25
                if dtype == torch.float16:
                    tol = tol + p.amax(1, keepdim=True) * v[:end].abs().sum(0) * 2.0 ** -36
                err = (out[i, r, hs].double() - o).abs()
                assert (err <= tol).all(), ("out", i, h, r, (err / tol).max().item(), o.abs().min().item())
                err = (lse[i, r, hs].double() - z[:, 0]).abs()
                assert (err <= (ds + 2.0 ** -20 + chain)[:, 0] + z[:, 0].abs() * 2.0 ** -22).all(), ("lse", i, h, r, err.max().item())
                total[: end - prefix] += p[:, prefix:].sum(0)
                total_tol[: end - prefix] += (p[:, prefix:] * (2 * rel + chain)).sum(0)
            err = (w[i, h].double() - total).abs()
            assert (err <= total_tol + total.abs() * (rows * grp + 2) * 2.0 ** -24).all(), ("weights", i, h, err.max().item())
