"""What the operators around a batch's KV cache are measured on: rotary positions, attention behind a shared prefix, eviction.

Three operators of one serving loop: new queries and keys are rotated (cass_rope), every sequence attends to a prompt that all of
them share and to its own cache, and the weights that its positions get are summed (cass_shared_prefix_attention); a cache that
has grown beyond its budget keeps the positions with the largest sums (cass_kv_evict).

Every operator has a plain form in elementary torch operations (`own` false) and the library's entry point (`own` true).
Queries and keys are N(0, 1) with 2 % of the keys' channels x4; prompts' keys have a few positions that all queries favour, as
trained models have.
"""
from __future__ import annotations

import math
import random
import types

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HEADS = {           # query heads, KV heads, head size: the benchmark's configurations
    "tiny": (4, 2, 64),
    "llama8b": (32, 8, 128),
    "qwen": (40, 8, 128),
}
ROPE_VALUES = 32768 * 48 * 128         # most values of a drawn rotation
PREFIX_ROWS = 64 * 32768               # most (sequence, prefix position) pairs of a drawn attention
CACHE_ROWS = 65536                     # most cache positions over all sequences of a drawn case


def listed():
    return [
        # one token of the tiny model: the call itself
        dict(name="rope_tiny_1", op="rope", heads="tiny", rot=64, rows=1, type="bf16", layout="half", scaling="none", factor=1.0,
             transpose=False, packed=True, start=300),
        # gamma + 1 = 5 rows of 8 sequences, q and k inside the projection's packed rows, a model stretched for long contexts
        dict(name="rope_8b_8x5", op="rope", heads="llama8b", rot=128, rows=40, type="bf16", layout="half", scaling="bands", factor=8.0,
             transpose=False, packed=True, start=100000),
        # a prompt of odd length, interleaved pairs in half of the head
        dict(name="rope_8b_prompt_8191", op="rope", heads="llama8b", rot=64, rows=8191, type="fp16", layout="interleaved", scaling="yarn",
             factor=4.0, transpose=False, packed=False, start=0),
        # the gradient of 32768 rows in training, 32-bit values
        dict(name="rope_qwen_gradient_32768", op="rope", heads="qwen", rot=128, rows=32768, type="fp32", layout="half", scaling="none",
             factor=1.0, transpose=True, packed=False, start=0),
        # two short sequences of the tiny model: launches and little else
        dict(name="attend_tiny_2", op="attend", heads="tiny", batch=2, rows=1, prefix=100, cap=33, lens=1, type="bf16", order="bphd", weights=False),
        # eight chats behind a system prompt, one new token each
        dict(name="attend_8b_8x1_4000", op="attend", heads="llama8b", batch=8, rows=1, prefix=4000, cap=600, lens=2, type="bf16", order="bphd",
             weights=False),
        # verification of gamma + 1 = 5 drafted rows of 16 sequences behind a long document, weights summed for eviction
        dict(name="attend_8b_16x5_16000", op="attend", heads="llama8b", batch=16, rows=5, prefix=16000, cap=1023, lens=3, type="bf16",
             order="bphd", weights=True),
        # one sequence without a prefix, a long cache of its own, weights summed
        dict(name="attend_8b_1x1_own_32000", op="attend", heads="llama8b", batch=1, rows=1, prefix=0, cap=32000, lens=4, type="bf16",
             order="bhpd", weights=True),
        # many sequences behind a very long prefix: the products count
        dict(name="attend_qwen_64x1_32768", op="attend", heads="qwen", batch=64, rows=1, prefix=32768, cap=1000, lens=5, type="fp16",
             order="bphd", weights=False),
        # one sequence a little over its budget, as after every hundred tokens of a decode
        dict(name="evict_8b_1x1152", op="evict", heads="llama8b", batch=1, cap=1152, lens=6, budget=1024, first=4, last=256, type="bf16",
             order="bphd"),
        # eight sequences cut to half
        dict(name="evict_qwen_8x4095", op="evict", heads="qwen", batch=8, cap=4095, lens=7, budget=2000, first=4, last=128, type="fp16",
             order="bphd"),
        # long prompts cut to what matters
        dict(name="evict_8b_4x32768", op="evict", heads="llama8b", batch=4, cap=32768, lens=8, budget=4096, first=16, last=512, type="bf16",
             order="bhpd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "attend", "attend", "evict"))
    heads = rng.choice(("tiny", "llama8b", "llama8b", "qwen"))
    nq, nk, d = HEADS[heads]
    if op == "rope":
        scaling = rng.choice(("none", "linear", "ntk", "bands", "yarn"))
        return dict(op=op, heads=heads, rot=rng.choice((d, d, d // 2, 2 * rng.randint(2, d // 2))), rows=_log_int(rng, 1, ROPE_VALUES // ((nq + nk) * d)),
                    type=rng.choice(tuple(TYPES)), layout=rng.choice(("half", "interleaved")), scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)), transpose=rng.random() < 0.3,
                    packed=rng.random() < 0.5, start=rng.choice((0, _log_int(rng, 1, 1000000))))
    batch = _log_int(rng, 1, 64)
    cap = _log_int(rng, 16, CACHE_ROWS // batch)
    case = dict(op=op, heads=heads, batch=batch, cap=cap, lens=rng.randrange(1 << 30), type=rng.choice(("bf16", "bf16", "fp16")),
                order=rng.choice(("bphd", "bphd", "bhpd")))
    if op == "attend":
        case.update(rows=rng.choice((1, 1, 1, 2, 5, 7, 16)), weights=rng.random() < 0.4)
        prefix = PREFIX_ROWS // (batch * case["rows"])
        case["prefix"] = 0 if rng.random() < 0.15 else _log_int(rng, 16, min(65536, prefix))
        return case
    budget = max(8, int(cap * rng.uniform(0.1, 0.95)))
    case.update(budget=budget, first=rng.choice((0, 1, 4)), last=min(rng.choice((0, 16, 128, 500)), budget // 2))
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *size):
    return torch.randn(*size, generator=g, device=DEV, dtype=torch.float32)


def _lens(case):
    """Lengths of the sequences' caches: most of the room for one sequence, from a half of it up for more; they follow from the case."""
    rng, cap, need = random.Random(case["lens"]), case["cap"], case.get("rows", 1)
    if case["batch"] == 1:
        return [max(need, cap - rng.randint(0, cap // 64))] if case["op"] == "attend" else [cap]
    return [max(min(need, cap), rng.randint(cap // 2, cap)) for _ in range(case["batch"])]


def _keys(g, n, heads, d, dtype):
    k = _normal(g, n, heads, d)
    k[:, :, torch.randperm(d, generator=g, device=DEV)[: max(1, d // 50)]] *= 4.0
    return k.to(dtype)


def _in_order(x, order):
    """[batch][position][head][dim], stored in that order or with the heads before the positions."""
    return x if order == "bphd" else x.transpose(1, 2).contiguous().transpose(1, 2)


def _caches(g, case):
    _, nk, d = HEADS[case["heads"]]
    n, dtype = case["batch"] * case["cap"], TYPES[case["type"]]
    k = _keys(g, n, nk, d, dtype).view(case["batch"], case["cap"], nk, d)
    v = _normal(g, case["batch"], case["cap"], nk, d).to(dtype)
    return _in_order(k, case["order"]), _in_order(v, case["order"])


ROPE_TRAINED = 8192                    # positions that the scaled frequencies' model was trained on
ROPE_THETA = 500000.0
BANDS_LOW, BANDS_HIGH = 1.0, 4.0       # wavelengths above trained / low are stretched, those below trained / high are not
YARN_SLOW, YARN_FAST = 1.0, 32.0       # rotations within the trained positions between which the stretching fades out


def _frequencies(case):
    """64-bit angle per position of every pair, and the factor on sines and cosines."""
    rot, s, kind = case["rot"], case["factor"], case["scaling"]
    j = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    theta = ROPE_THETA * s ** (rot / (rot - 2)) if kind == "ntk" else ROPE_THETA
    f = theta ** (-2.0 * j / rot)
    if kind == "linear":
        f = f / s
    elif kind == "bands":
        wave = 2 * math.pi / f
        mix = ((ROPE_TRAINED / wave - BANDS_LOW) / (BANDS_HIGH - BANDS_LOW)).clamp(0, 1)
        f = (1 - mix) * f / s + mix * f
    elif kind == "yarn":
        at = lambda beta: rot * math.log(ROPE_TRAINED / (2 * math.pi * beta)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(YARN_FAST)), 0), min(math.ceil(at(YARN_SLOW)), rot - 1)
        ramp = ((j - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = ramp * f / s + (1 - ramp) * f
    return f, 0.1 * math.log(s) + 1 if kind == "yarn" else 1.0


def _strides(t, *dims):
    return [t.stride(i) for i in dims]


def _inputs(case, seed):
    g, (nq, nk, d) = _gen(seed), HEADS[case["heads"]]
    s, dtype = types.SimpleNamespace(case=case), TYPES[case["type"]]
    if case["op"] == "rope":
        rows = case["rows"]
        if case["packed"]:
            # q, k and v rows of one projection: what is rotated lies inside
            qkv = _normal(g, rows, nq + 2 * nk, d).to(dtype)
            s.q, s.k = qkv[:, :nq], qkv[:, nq: nq + nk]
        else:
            s.q, s.k = _normal(g, rows, nq, d).to(dtype), _normal(g, rows, nk, d).to(dtype)
        first = torch.randint(case["start"], case["start"] + 1000, (1,), generator=g, device=DEV)
        s.pos = (first + torch.arange(rows, device=DEV)).to(torch.int32)
        if rows <= 64:                                     # a few rows of several sequences: positions of their own
            s.pos = s.pos + 17 * torch.randint(0, 1000, (rows,), generator=g, device=DEV, dtype=torch.int32)
        s.q_out, s.k_out = (torch.zeros(rows, n, d, dtype=dtype, device=DEV) for n in (nq, nk))
    elif case["op"] == "attend":
        s.q = _normal(g, case["batch"], case["rows"], nq, d).mul_(1.5).to(dtype)
        s.kp = _keys(g, case["prefix"], nk, d, dtype)
        s.vp = _normal(g, case["prefix"], nk, d).to(dtype)
        s.kc, s.vc = _caches(g, case)
        s.lens = torch.tensor(_lens(case), dtype=torch.int32, device=DEV)
        s.out = torch.zeros_like(s.q)
        s.lse = torch.zeros(case["batch"], case["rows"], nq, device=DEV)
        s.w_in = s.w_out = None
        if case["weights"]:
            s.w_in = torch.rand(case["batch"], nk, case["cap"], generator=g, device=DEV)
            s.w_out = torch.zeros_like(s.w_in)
    else:
        s.kc, s.vc = _caches(g, case)
        # sums of attention weights: a few positions have most, many have nothing and tie
        w = torch.exp(_normal(g, case["batch"], nk, case["cap"]).mul_(2.0).sub_(4.0))
        s.w = torch.where(w < 0.005, torch.zeros_like(w), w)
        s.lens = torch.tensor(_lens(case), dtype=torch.int32, device=DEV)
        s.k_out, s.v_out = (_in_order(torch.zeros(case["batch"], case["budget"], nk, d, dtype=dtype, device=DEV), case["order"]) for _ in range(2))
        s.w_out = torch.zeros(case["batch"], nk, case["budget"], device=DEV)
        s.kept = torch.zeros(case["batch"], nk, case["budget"], dtype=torch.int32, device=DEV)
        s.new_lens = torch.zeros_like(s.lens)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _keep(s)
    elif case["op"] == "rope":
        s.freqs, s.gain = _frequencies(case)
    return s


def _keep(s):
    """What a user of the library keeps between calls: frequencies, descriptions of the layouts, scratch."""
    from paper_2605_26558_b200 import binding as B
    case, (nq, nk, d) = s.case, HEADS[s.case["heads"]]
    s.B = B
    dtype = {"bf16": B.BF16, "fp16": B.F16, "fp32": B.F32}[case["type"]]
    if case["op"] == "rope":
        kind = {"none": B.ROPE_PLAIN, "linear": B.ROPE_LINEAR, "ntk": B.ROPE_NTK, "bands": B.ROPE_BANDS, "yarn": B.ROPE_YARN}[case["scaling"]]
        low, high = (BANDS_LOW, BANDS_HIGH) if case["scaling"] == "bands" else (YARN_SLOW, YARN_FAST)
        s.freqs = torch.zeros(case["rot"] // 2 + 1, dtype=torch.float64, device=DEV)
        B.cass_rope_freqs(B.RopeParams(case["rot"], kind, ROPE_THETA, case["factor"], low, high, ROPE_TRAINED, 0.0), s.freqs)
        s.geom = B.RopeGeom(dtype, d, case["rot"], int(case["layout"] == "interleaved"), nq, nk, *_strides(s.q, 0, 1), *_strides(s.k, 0, 1),
                            *_strides(s.q_out, 0, 1), *_strides(s.k_out, 0, 1))
    else:
        s.geom = B.CacheGeom(dtype, case["batch"], nk, d, case["cap"], *_strides(s.kc, 0, 1, 2))
        if case["op"] == "attend":
            s.attn = B.SharedAttn(nq, case["rows"], *_strides(s.q, 0, 1, 2), *_strides(s.out, 0, 1, 2), case["prefix"], *_strides(s.kp, 0, 1), 0.0)
            s.scratch = torch.zeros(B.cass_shared_prefix_scratch_bytes(s.geom, s.attn, case["weights"]), dtype=torch.uint8, device=DEV)
            s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        else:
            s.geom_out = B.CacheGeom(dtype, case["batch"], nk, d, case["budget"], *_strides(s.k_out, 0, 1, 2))


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    return {"rope": _rope, "attend": _attend, "evict": _evict}[s.case["op"]](s)


def _rope(s):
    case = s.case
    if own:
        s.B.cass_rope(s.geom, s.freqs, s.pos, case["rows"], s.q.data_ptr(), s.k.data_ptr(), s.q_out, s.k_out, int(case["transpose"]))
        return s.q_out, s.k_out
    rot, half = case["rot"], case["rot"] // 2
    angle = s.pos.double()[:, None] * s.freqs
    c, sn = (angle.cos() * s.gain).float()[:, None], (angle.sin() * s.gain).float()[:, None]
    if case["transpose"]:
        sn = -sn

    def rotate(x):
        y = x.float()
        a, b = (y[..., :half], y[..., half:rot]) if case["layout"] == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
        r = (a * c - b * sn, a * sn + b * c)
        head = torch.cat(r, dim=-1) if case["layout"] == "half" else torch.stack(r, dim=-1).flatten(-2)
        return torch.cat((head, y[..., rot:]), dim=-1).to(x.dtype)

    return rotate(s.q), rotate(s.k)


def _attend(s):
    case, (nq, nk, d) = s.case, HEADS[s.case["heads"]]
    outputs = lambda out, lse, w: (out, lse, w) if case["weights"] else (out, lse)  # noqa: E731
    if own:
        s.B.cass_shared_prefix_attention(s.geom, s.attn, s.q, s.kp, s.vp, s.kc.data_ptr(), s.vc.data_ptr(), s.lens, s.out, s.lse, s.w_in,
                                         s.w_out, s.scratch, s.scratch.numel(), s.status)
        return outputs(s.out, s.lse, s.w_out)
    batch, rows, cap, grp = case["batch"], case["rows"], case["cap"], nq // nk
    q = s.q.float().view(batch, rows, nk, grp, d).permute(2, 0, 1, 3, 4) / math.sqrt(d)           # [head][sequence][row][in group][dim]
    qf = q.reshape(nk, batch * rows * grp, d)
    sp = (qf @ s.kp.float().permute(1, 2, 0)).view(nk, batch, rows, grp, case["prefix"])
    qs = q.permute(1, 0, 2, 3, 4).reshape(batch, nk, rows * grp, d)
    sc = (qs @ s.kc.float().permute(0, 2, 3, 1)).view(batch, nk, rows, grp, cap)
    at = torch.arange(cap, device=DEV)
    seen = at[None, None, :] < (s.lens[:, None] - (rows - 1 - torch.arange(rows, device=DEV)))[:, :, None]     # [sequence][row][position]
    sc = torch.where(seen[:, None, :, None, :], sc, torch.full_like(sc, -math.inf))
    m = sc.amax(dim=-1)
    if case["prefix"]:
        m = torch.maximum(m, sp.amax(dim=-1).transpose(0, 1))
    ps, pp = torch.exp(sc - m[..., None]), torch.exp(sp - m.transpose(0, 1)[..., None])
    total = ps.sum(dim=-1) + pp.sum(dim=-1).transpose(0, 1)                                        # [sequence][head][row][in group]
    live = (at[None, :] < s.lens[:, None])[:, :, None, None]
    o = ps.view(batch, nk, rows * grp, cap) @ torch.where(live, s.vc.float(), torch.zeros((), device=DEV)).permute(0, 2, 1, 3)
    o = o.view(batch, nk, rows, grp, d)
    o = o + (pp.view(nk, batch * rows * grp, -1) @ s.vp.float().transpose(0, 1)).view(nk, batch, rows, grp, d).transpose(0, 1)
    o = (o / total[..., None]).permute(0, 2, 1, 3, 4).reshape(batch, rows, nq, d).to(s.q.dtype)
    lse = (m + total.log()).permute(0, 2, 1, 3).reshape(batch, rows, nq)
    return outputs(o, lse, s.w_in + (ps / total[..., None]).sum(dim=(2, 3)) if case["weights"] else None)


def _evict(s):
    case = s.case
    if own:
        s.B.cass_kv_evict(s.geom, s.kc.data_ptr(), s.vc.data_ptr(), s.w, s.lens, case["budget"], case["first"], case["last"], s.geom_out,
                          s.k_out.data_ptr(), s.v_out.data_ptr(), s.w_out, s.kept, s.new_lens)
        return s.kept, s.new_lens, s.w_out, s.k_out, s.v_out
    cap, budget, n = case["cap"], case["budget"], s.lens[:, None, None]
    at = torch.arange(cap, device=DEV).expand_as(s.w)
    stays = (at < case["first"]) | (at >= n - case["last"]) | (n <= budget)
    rank = torch.where(stays, torch.full_like(s.w, math.inf), s.w)
    rank = torch.where(at < n, rank, torch.full_like(rank, -math.inf))
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]            # ties: the lower position first
    count = torch.minimum(s.lens, torch.full_like(s.lens, budget))
    there = torch.arange(budget, device=DEV) < count[:, None, None]
    kept = torch.sort(torch.where(there, best, torch.full_like(best, cap)), dim=-1).values
    take = kept.clamp(max=cap - 1)
    w = torch.where(there, torch.gather(s.w, 2, take), torch.zeros((), device=DEV))
    rows = take.transpose(1, 2)[..., None].expand(-1, -1, -1, s.kc.shape[3])
    live = there.expand(-1, s.w.shape[1], -1).transpose(1, 2)[..., None]
    k, v = (torch.where(live, torch.gather(x, 1, rows), torch.zeros((), dtype=x.dtype, device=DEV)) for x in (s.kc, s.vc))
    return torch.where(there, kept, -torch.ones_like(kept)).to(torch.int32), count, w, k, v


# ---- definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](s)


def _exact_rope(s):
    case, rot = s.case, s.case["rot"]
    f, gain, factor = [], 1.0, case["factor"]
    for j in range(rot // 2):
        x = ROPE_THETA ** (-2.0 * j / rot)
        if case["scaling"] == "linear":
            x /= factor
        elif case["scaling"] == "ntk":
            x = (ROPE_THETA * factor ** (rot / (rot - 2.0))) ** (-2.0 * j / rot)
        elif case["scaling"] == "bands":
            turns = ROPE_TRAINED * x / (2 * math.pi)                # over the trained positions
            if turns < BANDS_LOW:
                x /= factor
            elif turns <= BANDS_HIGH:
                t = (turns - BANDS_LOW) / (BANDS_HIGH - BANDS_LOW)
                x = x * (t + (1 - t) / factor)
        elif case["scaling"] == "yarn":
            pair = [rot * math.log(ROPE_TRAINED / (2 * math.pi * beta)) / (2 * math.log(ROPE_THETA)) for beta in (YARN_FAST, YARN_SLOW)]
            lo, hi = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), rot - 1)
            t = min(max((j - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            x = x * (1 - t + t / factor)
        f.append(x)
    if case["scaling"] == "yarn":
        gain = 1 + 0.1 * math.log(factor)
    angle = s.pos.double()[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, gain), -angle if case["transpose"] else angle)[:, None]
    out = []
    for x in (s.q, s.k):
        y = x.double()
        if case["layout"] == "half":
            z = torch.complex(y[..., : rot // 2], y[..., rot // 2: rot]) * turn
            y[..., : rot // 2], y[..., rot // 2: rot] = z.real, z.imag
        else:
            z = torch.view_as_complex(y[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * turn
            y[..., :rot] = torch.view_as_real(z).flatten(-2)
        out.append(y)
    return tuple(out)


def _exact_attend(s):
    case, (nq, nk, d) = s.case, HEADS[s.case["heads"]]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s.lse.shape, dtype=torch.float64, device=DEV)
    w = s.w_in.double().clone() if case["weights"] else None
    for h in range(nk):
        kp, vp = s.kp[:, h].double(), s.vp[:, h].double()
        heads = range(h * (nq // nk), (h + 1) * (nq // nk))
        for b, n in enumerate(_lens(case)):
            k, v = torch.cat((kp, s.kc[b, :n, h].double())), torch.cat((vp, s.vc[b, :n, h].double()))
            for r in range(case["rows"]):
                hidden = case["rows"] - 1 - r                       # positions at the end that this row does not see
                end = case["prefix"] + max(n - hidden, 0)
                x = s.q[b, r, heads[0]: heads[-1] + 1].double() @ k[:end].T * d ** -0.5
                z = torch.logsumexp(x, dim=1, keepdim=True)
                p = torch.exp(x - z)
                lse[b, r, heads[0]: heads[-1] + 1] = z[:, 0]
                out[b, r, heads[0]: heads[-1] + 1] = p @ v[:end]
                if case["weights"]:
                    w[b, h, : end - case["prefix"]] += p[:, case["prefix"]:].sum(dim=0)
    return (out, lse, w) if case["weights"] else (out, lse)


def _exact_evict(s):
    case, weights, lens = s.case, s.w.cpu().tolist(), _lens(s.case)
    batch, _, nk, d = s.kc.shape
    budget = case["budget"]
    kept = torch.full((batch, nk, budget), -1, dtype=torch.int32)
    w = torch.zeros(batch, nk, budget, dtype=torch.float64)
    k, v = (torch.zeros(batch, budget, nk, d, dtype=torch.float64, device=DEV) for _ in range(2))
    for b, n in enumerate(lens):
        for h in range(nk):
            stay = list(range(n))
            if n > budget:
                edge = list(range(case["first"])) + list(range(n - case["last"], n))
                middle = sorted(range(case["first"], n - case["last"]), key=lambda j: (-weights[b][h][j], j))
                stay = sorted(edge + middle[: budget - len(edge)])
            kept[b, h, : len(stay)] = torch.tensor(stay, dtype=torch.int32)
            w[b, h, : len(stay)] = torch.tensor([weights[b][h][j] for j in stay], dtype=torch.float64)
            at = torch.tensor(stay, device=DEV)
            k[b, : len(stay), h], v[b, : len(stay), h] = s.kc[b, at, h].double(), s.vc[b, at, h].double()
    return kept.to(DEV), torch.tensor([min(n, budget) for n in lens], dtype=torch.int32, device=DEV), w.to(DEV), k, v


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    nq, nk, d = HEADS[case["heads"]]
    size = 4 if case["type"] == "fp32" else 2
    if case["op"] == "rope":
        values = case["rows"] * (nq + nk) * d
        return dict(bytes=2 * values * size + 4 * case["rows"], flops=3 * case["rows"] * (nq + nk) * case["rot"])
    lens = _lens(case)
    if case["op"] == "attend":
        rows = case["batch"] * case["rows"]
        seen = rows * case["prefix"] + sum(max(n - r, 0) for n in lens for r in range(case["rows"]))
        moved = 2 * (case["prefix"] + sum(lens)) * nk * d * size + 2 * rows * nq * d * size + 4 * rows * nq
        return dict(bytes=moved + (8 * case["batch"] * nk * case["cap"] if case["weights"] else 0), flops=4 * seen * nq * d)
    stay = sum(min(n, case["budget"]) for n in lens)
    return dict(bytes=nk * (4 * sum(lens) + 4 * stay * d * size + 8 * case["batch"] * case["budget"]), flops=0)
