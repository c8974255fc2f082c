"""The operators that serve prompts in chunks from a paged cache of 4 or 8 bits and keep it within a budget, and the cases that their speed
and results are followed on.

  chunk   attn_cache_chunk_fwd    attention of chunks of new tokens, packed, one chunk per sequence, over the cache
  weigh   attn_cache_weigh        the attention weight that every cached key had from these queries, added to its sum
  evict   attn_cache_evict        the rows of least weight leave the cache, which is closed up in place

Where `own` is false the same is computed in elementary torch operations in 32 bits (sums of weights over the queries in 64).

The cache: codes k, v [pages, Hkv, page, d * bits / 8] and one scale byte per 32 channels; key j of sequence b is in page
table[b, j / page] at j % page.  4 bits: e2m1 codes, the even channel in the low half of a byte; 8 bits: e4m3 codes; a scale byte s stands for
2^(s - 127).  Weights: fp32 [pages, Hkv, page], one per row of the cache.
"""
import math
import random

import numpy as np
import torch

own = False

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_HEADS = {"H": 32, "Hkv": 8, "dqk": 128, "dv": 128, "bits": 4, "page": 64, "dtype": "bf16"}


def _chunk(name, B, qlo, qhi, lo, hi, **more):
    """B sequences with qlo ... qhi new tokens (the first `single` of them with one, the last `idle` with none) behind lo ... hi cached ones
    (`causal`; otherwise the keys are lo ... hi, and the queries no part of them); `pad` rows behind the last sequence."""
    return {"name": name, "kind": "chunk", "B": B, "qlo": qlo, "qhi": qhi, "lo": lo, "hi": hi, "single": 0, "idle": 0, "pad": 0, "causal": True,
            "len_seed": 0, **_HEADS, **more}


def _weigh(name, B, qlo, qhi, lo, hi, packed, **more):
    """Lengths as in _chunk; packed = False: the [B, Nq, heads, d] queries of a decode step (qlo = qhi)."""
    return {**_chunk(name, B, qlo, qhi, lo, hi), "kind": "weigh", "packed": packed, **more}


def _evict(name, B, lo, hi, keep, recent, **more):
    """B sequences of lo ... hi rows, of which `keep` are to stay, the last `recent` among them."""
    return {"name": name, "kind": "evict", "B": B, "lo": lo, "hi": hi, "keep": keep, "recent": recent, "len_seed": 0, **_HEADS, **more}


def listed():
    return [
        # the rest of one prompt behind a shared prefix: latency
        _chunk("chunk_T16_N500", 1, 16, 16, 484, 484),
        # a chunk of a long prompt against what is cached of it
        _chunk("chunk_T2048_N30001", 1, 2048, 2048, 27953, 27953),
        # whole prompts of different lengths, nothing cached yet, 8 bits
        _chunk("chunk_prompts_B4_8bit", 4, 300, 4000, 0, 0, bits=8, len_seed=5),
        # a continuous batch: requests that decode, two chunks of prompts, slots without a request, a padded batch
        _chunk("chunk_mixed_B26", 26, 128, 256, 100, 4096, single=22, idle=2, pad=37, page=16, len_seed=3),
        # decoder queries over an encoder's memory: no mask, heads of their own, fp16
        _chunk("chunk_cross_d64_8bit_fp16", 16, 1, 50, 1500, 1500, H=12, Hkv=12, dqk=64, dv=64, bits=8, page=32, causal=False, dtype="fp16"),
        # a decode step of 32 requests of equal lengths: its weights
        _weigh("weigh_decode_B32_N4001", 32, 1, 1, 4000, 4000, False, page=16),
        # a chunk of a prompt over 16 001 keys
        _weigh("weigh_chunk_T1024_N16001", 1, 1024, 1024, 14977, 14977, True),
        # a few drafted tokens of four requests, small heads, 8 bits, fp16: latency
        _weigh("weigh_draft_d64_8bit_fp16", 4, 1, 8, 30, 600, True, H=16, Hkv=4, dqk=64, dv=64, bits=8, page=32, dtype="fp16", len_seed=2),
        # requests that decoded 256 tokens past their budget
        _evict("evict_decode_B32", 32, 4352, 4352, 4096, 64),
        # a long prompt, all of it cached, cut down to its budget
        _evict("evict_prompt_N30001", 1, 30001, 30001, 4096, 128),
        # a few short requests, some within their budget, 8 bits: latency
        _evict("evict_small_8bit", 3, 100, 400, 128, 32, bits=8, page=16, len_seed=1),
    ]


DIMS = [(64, 64), (96, 96), (128, 128), (192, 128), (256, 256)]


def draw(rng):
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        Hkv = rng.choice([1, 2, 4, 8, 8, 16])
        H = Hkv * rng.choice([1, 2, 4, 4, 8])
        dqk, dv = rng.choice(DIMS + [(128, 128), (128, 128)])
        if H > 64:
            continue
        heads = {"H": H, "Hkv": Hkv, "dqk": dqk, "dv": dv, "bits": rng.choice([4, 4, 8]), "page": 1 << rng.randint(4, 8),
                 "dtype": "fp16" if rng.random() < 0.3 else "bf16", "len_seed": rng.randrange(1 << 20)}
        B = logu(1, 64)
        kind = rng.choice(["chunk", "chunk", "chunk", "weigh", "weigh", "evict", "evict"])
        if kind == "evict":
            hi = logu(16, 32000)
            lo = hi if rng.random() < 0.3 else max(1, hi // rng.choice([2, 8, 64]))
            keep = logu(1, hi)
            c = _evict("", B, lo, hi, keep, rng.choice([0, 1, 16, 64, 200, keep]), **heads)
        else:
            hi, qhi = logu(16, 32000), logu(1, 2048)
            lo = hi if rng.random() < 0.3 else max(1, hi // rng.choice([2, 8, 64]))
            qlo = qhi if rng.random() < 0.3 else max(1, qhi // rng.choice([2, 8, 64]))
            idle = rng.randint(0, B // 4)
            more = dict(heads, causal=rng.random() < 0.8, single=rng.choice([0, 0, (B - idle) // 2]), idle=idle)
            if rng.random() < 0.2:
                lo = hi = 0
                more["causal"] = True
            if kind == "chunk":
                c = _chunk("", B, qlo, qhi, lo, hi, pad=rng.choice([0, 0, 5, 100]), **more)
            elif rng.random() < 0.5:
                c = _weigh("", B, qlo, qhi, lo, hi, True, **more)
            else:
                qhi = min(qhi, rng.choice([1, 1, 4, 8]))
                c = _weigh("", B, qhi, qhi, lo, hi, False, **dict(more, single=0, idle=0))
            # the plain form holds all scores of sequences as long as the longest
            if B * H * qhi * (hi + qhi) > 2.0e9 or B * Hkv * (hi + qhi) * (dqk + dv) > 6e8:
                continue
        w = work(c)
        if 2e3 <= w["bytes"] <= 3.2e8 and w["flops"] <= 9.5e11:
            del c["name"]
            return c


def _lengths(case):
    """(queries, keys) of every sequence, log-uniform in the case's ranges."""
    r = random.Random(case["len_seed"])
    logu = lambda lo, hi: int(round(math.exp(r.uniform(math.log(lo), math.log(hi))))) if hi > 0 else 0
    B = case["B"]
    cached = [logu(case["lo"], case["hi"]) for _ in range(B)]
    if case["kind"] == "evict":
        return [0] * B, cached
    new = [1 if b < case["single"] else 0 if b >= B - case["idle"] else logu(case["qlo"], case["qhi"]) for b in range(B)]
    return new, [c + n if case["causal"] else c for c, n in zip(cached, new)]


def _pairs(nq, n, causal):
    """Visible (query, key) pairs of a sequence; the last query is aligned with the last key."""
    return sum(range(n - nq + 1, n + 1)) if causal else nq * n


def work(case):
    new, lens = _lengths(case)
    H, Hkv, dqk, dv, bits = (case[n] for n in ("H", "Hkv", "dqk", "dv", "bits"))
    row = lambda d: d * bits // 8 + d // 32
    if case["kind"] == "evict":
        moved = read = 0
        for n in lens:
            if n > case["keep"]:
                recent = min(case["recent"], case["keep"])
                stay, of = case["keep"] - recent, n - recent               # of weights in no order, a share of the rows that stay lies behind
                moved += recent + stay * (of - stay) / of
                read += n
        return {"bytes": int(Hkv * (4 * read + 2 * moved * (row(dqk) + row(dv) + 4))) + 12 * case["B"], "flops": 4 * Hkv * read}
    pairs = sum(_pairs(nq, n, case["causal"]) for nq, n in zip(new, lens))
    keys, T = sum(n for nq, n in zip(new, lens) if nq), sum(new)
    if case["kind"] == "chunk":
        return {"bytes": keys * Hkv * (row(dqk) + row(dv)) + T * H * (2 * (dqk + dv) + 4), "flops": 2 * pairs * H * (dqk + dv)}
    return {"bytes": keys * Hkv * (row(dqk) + 8) + T * H * (2 * dqk + 4), "flops": 2 * pairs * H * dqk}


# ---------------------------------------------------------------------------------------------------------------------------
# the plain forms

def _values(raw, scale, bits):
    """The numbers, in 32 bits, of rows of codes [..., d * bits / 8] with scale bytes [..., d / 32]."""
    if bits == 4:
        code = torch.stack((raw & 15, raw >> 4), dim=-1).flatten(-2)
        v = torch.tensor(_E2M1, device=raw.device)[(code & 7).long()]
        v = torch.where(code >= 8, -v, v)
    else:
        v = raw.view(torch.float8_e4m3fn).float()
    return torch.ldexp(v.unflatten(-1, (-1, 32)), (scale.int() - 127)[..., None]).flatten(-2)


def _slots(s, longest):
    """Slots [B, longest] of the sequences' keys (behind the last one: some slot of theirs)."""
    page = s["cache"][0].shape[2]
    j = torch.arange(longest, device="cuda")
    return s["table"].long()[:, j // page] * page + j % page


def _scores(s):
    """Scores [B, Hkv, Nq, G, N] in 32 bits, -inf where a query does not see a key, of the batch padded to its longest chunk and sequence; and
    the row of q [B, Nq] that a query is, and whether there is one."""
    q, B, N, Nq = s["q"], s["lens"].shape[0], s["longest"], s["most_queries"]
    kc, ks = s["cache"][:2]
    Hkv, page = kc.shape[1], kc.shape[2]
    first, new = s["cu"][:-1].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    i = torch.arange(Nq, device="cuda")
    there = i < new[:, None]
    row = torch.where(there, first[:, None] + i, 0)
    G, d = q.shape[1] // Hkv, q.shape[2]
    slots = _slots(s, N)
    k = _values(kc[slots // page, :, slots % page], ks[slots // page, :, slots % page], s["bits"]).permute(0, 2, 3, 1).contiguous()
    qg = q[row].float().reshape(B, Nq, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Nq * G, d)
    sc = torch.matmul(qg, k).mul_(s["scale"]).view(B, Hkv, Nq, G, N)
    lens = s["lens"].long()[:, None]
    last = lens - new[:, None] + i if s["causal"] else lens - 1 + 0 * i
    seen = (torch.arange(N, device="cuda") <= last[:, :, None]) & there[:, :, None]
    return sc.masked_fill_(~seen[:, None, :, None, :], -math.inf), row, there


def _row_sums(sc):
    """exp(scores - maximum), in place, the sums of its rows and the rows' log-sum-exp."""
    m = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return p, l, torch.where(l > 0, m + torch.log(l), -math.inf)


def _unpad(x, s):
    """Rows [T, ...] of a padded batch [B, Nq, ...]; zeros behind the last sequence."""
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    held = b < s["lens"].shape[0]
    b = torch.where(held, b, 0)
    i = torch.where(held, t - s["cu"].long()[b], 0)
    y = x[b, i]
    return torch.where(held.view(-1, *[1] * (y.dim() - 1)), y, 0.0)


def _plain_chunk(s):
    sc, _, _ = _scores(s)
    B, Hkv, Nq, G, N = sc.shape
    p, l, lse = _row_sums(sc)
    vc, vs = s["cache"][2:]
    page, slots = vc.shape[2], _slots(s, N)
    v = _values(vc[slots // page, :, slots % page], vs[slots // page, :, slots % page], s["bits"]).transpose(1, 2).contiguous()
    o = torch.matmul(p.view(B, Hkv, Nq * G, N), v).view(B, Hkv, Nq, G, -1)
    o = torch.where(l > 0, o / l, 0.0).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return _unpad(o, s).to(s["q"].dtype), _unpad(lse[..., 0].permute(0, 2, 1, 3).flatten(2, 3), s).T.contiguous()


def _plain_weigh(s):
    sc, row, there = _scores(s)
    B, Hkv, Nq, G, N = sc.shape
    lse = s["lse_rows"][row].view(B, Nq, Hkv, G).permute(0, 2, 1, 3)[..., None]
    p = torch.exp(sc - torch.where(there[:, None, :, None, None], lse, 0.0))
    got = p.sum(dim=(2, 3), dtype=torch.float64).transpose(1, 2)                            # [B, N, Hkv]
    w, j = s["weights"], torch.arange(N, device="cuda")
    lens, new = s["lens"].long()[:, None], (s["cu"][1:] - s["cu"][:-1]).long()[:, None]
    at = torch.where(j < lens, j, 0)                                                         # behind the end: key 0 once more
    slots, page = _slots(s, N).gather(1, at), w.shape[2]
    old = w[slots // page, :, slots % page]
    fresh = (j >= lens - new) if s["fresh"] else torch.zeros_like(slots, dtype=torch.bool)
    sums = (torch.where(fresh[..., None], 0.0, old.double()) + got).float()
    sums = torch.where(((new > 0) & (lens > 0))[..., None], sums, old)
    w[slots // page, :, slots % page] = sums.gather(1, at[..., None].expand_as(sums))
    return w


def _plain_evict(s):
    w, (kc, ks, vc, vs), lens, keep = s["weights"], s["cache"], s["lens"].long(), s["keep"].long()
    Hkv, page, N = w.shape[1], w.shape[2], s["longest"]
    slots, j = _slots(s, N), torch.arange(N, device="cuda")
    p, at, h = (slots // page)[:, None, :], (slots % page)[:, None, :], torch.arange(Hkv, device="cuda")[:, None]
    full = (lens > keep)[:, None, None]
    left = torch.minimum(lens, keep.clamp(min=0))
    recent = left.clamp(max=s["recent"])[:, None, None]
    stay, of = left[:, None, None] - recent, lens[:, None, None] - recent                    # so many of the first `of` rows stay
    x = torch.where(j < of, w[p, h, at], -math.inf)                                          # [B, Hkv, N]
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order).contiguous())
    stays = (rank < stay) & (j < of)
    hole, mover = ~stays & (j < stay), stays & (j >= stay)
    movers = torch.sort(torch.where(mover, j, N), dim=-1).values                             # in their order
    src = torch.where(hole, movers.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)).clamp(max=N - 1), j)
    src = torch.where((j >= stay) & (j < stay + recent), j + (lens - left)[:, None, None], src).clamp(max=N - 1)
    src = torch.where(full & (j < left[:, None, None]), src, torch.where(j < lens[:, None, None], j, 0))
    src = torch.where(j < lens[:, None, None], src, src[..., :1])                            # behind the end: what row 0 gets
    to = torch.where(j < lens[:, None, None], j, 0)
    move = lambda t: t.index_put_((p.gather(-1, to[:, :1]), h, at.gather(-1, to[:, :1])),
                                  t[p.expand_as(src).gather(-1, src), h, at.expand_as(src).gather(-1, src)])
    return (left.int(), *(move(t) for t in (w, kc, ks, vc, vs)))


# ---------------------------------------------------------------------------------------------------------------------------

def _some_cache(case, pages, normal, gen):
    """A cache whose every slot holds values as a model's keys and values have them (N(0, 1), a few channels eight times that)."""
    Hkv, page, bits = case["Hkv"], case["page"], case["bits"]
    out = []
    for d in (case["dqk"], case["dv"]):
        outliers = torch.where(torch.rand(Hkv, 1, d, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
        codes = torch.empty(pages, Hkv, page, d * bits // 8, dtype=torch.uint8, device="cuda")
        scales = torch.empty(pages, Hkv, page, d // 32, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (Hkv * page * d))
        for i in range(0, pages, step):
            x = (normal(min(step, pages - i), Hkv, page, d) * outliers).unflatten(-1, (-1, 32))
            e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / (7.0 if bits == 4 else 448.0))).clamp(-100, 100)
            x = torch.ldexp(x, -e.int()).flatten(-2)
            if bits == 8:
                c = x.to(torch.float8_e4m3fn).view(torch.uint8)
            else:
                c = torch.bucketize(x.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")).to(torch.uint8)
                c = c + 8 * (x < 0).to(torch.uint8)
                c = c[..., 0::2] | (c[..., 1::2] << 4)
            codes[i:i + step], scales[i:i + step] = c, (e.squeeze(-1) + 127).to(torch.uint8)
        out += [codes, scales]
    return tuple(out)


def prepare(case, seed):
    dtype = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, dtype=torch.float32, device="cuda")
    new, lens = _lengths(case)
    B, page, Hkv = case["B"], case["page"], case["Hkv"]
    need = [max(1, (n + page - 1) // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").int()                       # pages as a server hands them out
    width = max(need)
    at = torch.tensor([sum(need[:b]) for b in range(B)], device="cuda")[:, None] + torch.arange(width, device="cuda")
    held = torch.arange(width, device="cuda") < torch.tensor(need, device="cuda")[:, None]
    table = order[at.clamp(max=pages - 1)]
    s = {"kind": case["kind"], "bits": case["bits"], "longest": max(1, *lens), "cache": _some_cache(case, pages, normal, gen)}
    s["table"] = torch.where(held, table, table[:, :1]).contiguous()
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["kind"] == "evict":
        # sums over many queries: over some orders of magnitude, the first keys' the largest; keys that hardly any query saw have equal ones
        w = torch.exp(1.5 * normal(pages, Hkv, page))
        w = torch.where(torch.rand(pages, Hkv, page, generator=gen, device="cuda") < 0.1, 2.0 ** -10, w)
        w[s["table"][:, 0].long(), :, :4] *= 1000.0
        s["weights"] = w
        s["keep"] = torch.full((B,), case["keep"], dtype=torch.int32, device="cuda")
        s["recent"] = case["recent"]
        return s
    cu = [sum(new[:b]) for b in range(B + 1)]
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    s["most_queries"] = max(1, *new)
    T = max(1, cu[-1] + (case["pad"] if case["kind"] == "chunk" else 0))
    s["q"] = normal(T, case["H"], case["dqk"]).to(dtype)
    s["scale"], s["causal"] = case["dqk"] ** -0.5, case["causal"]
    if case["kind"] == "chunk":
        s["o"], s["lse"] = torch.zeros(T, case["H"], case["dv"], dtype=dtype, device="cuda"), torch.zeros(case["H"], T, device="cuda")
        return s
    # the attention pass's log-sum-exp of every query, as that pass lays it out
    rows = _unpad(_row_sums(_scores(s)[0])[2][..., 0].permute(0, 2, 1, 3).flatten(2, 3), s)  # [T, H]
    s["packed"], s["lse_rows"] = case["packed"], rows
    s["lse"] = rows.T.contiguous() if case["packed"] else rows.view(B, case["qlo"], -1).transpose(1, 2).contiguous()
    s["weights"] = torch.exp(normal(pages, Hkv, page))
    s["fresh"] = case["causal"]
    return s


def run(s):
    if own:
        import paper_2603_05451_amd as A
        cache = A.AttnCache(*s["cache"])
        if s["kind"] == "chunk":
            return A.attn_cache_chunk_fwd(s["q"], cache, s["table"], s["cu"], s["lens"], s["scale"], s["causal"], o=s["o"], lse=s["lse"])
        if s["kind"] == "weigh":
            if s["packed"]:
                return A.attn_cache_weigh(s["q"], s["lse"], s["weights"], cache, s["table"], s["lens"], s["scale"], s["causal"], cu_seqlens=s["cu"],
                                          fresh=s["fresh"])
            B, H, Nq = s["lse"].shape
            return A.attn_cache_weigh(s["q"].view(B, Nq, H, -1), s["lse"], s["weights"], cache, s["table"], s["lens"], s["scale"], s["causal"],
                                      fresh=s["fresh"])
        # the cache comes back as its bytes, which are moved and stand for nothing else than before
        return (A.attn_cache_evict(s["weights"], cache, s["table"], s["lens"], s["keep"], s["recent"]), s["weights"], *s["cache"])
    if s["kind"] == "chunk":
        return _plain_chunk(s)
    return _plain_weigh(s) if s["kind"] == "weigh" else _plain_evict(s)


# ---------------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_rows(codes, scales, slots, head, bits):
    """Rows [len(slots), d] of one head."""
    page = codes.shape[2]
    if bits == 4:
        table = [m * sign for sign in (1.0, -1.0) for m in _E2M1]
    else:
        table = [sign * ((m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) if e * 8 + m < 127 else math.nan)
                 for sign in (1.0, -1.0) for e in range(16) for m in range(8)]
    table = torch.tensor(table, dtype=torch.float64, device="cuda")
    powers = torch.tensor([math.ldexp(1.0, i - 127) for i in range(255)] + [math.nan], dtype=torch.float64, device="cuda")
    raw = codes[slots // page, head, slots % page].long()
    x = table[raw] if bits == 8 else torch.stack((table[raw % 16], table[raw // 16]), -1).flatten(-2)
    return x * powers[scales[slots // page, head, slots % page].long()].repeat_interleave(32, -1)


def _exact_attention(case, s):
    """For every sequence and KV head: (sequence, head, slots, queries' rows, scores [queries, G, keys])."""
    new, lens = _lengths(case)
    G, page, first = case["H"] // case["Hkv"], case["page"], 0
    for b, (nq, n) in enumerate(zip(new, lens)):
        rows = torch.arange(first, first + nq, device="cuda")
        first += nq
        j = torch.arange(n, device="cuda")
        slots = s["table"][b, j // page].long() * page + j % page
        for h in range(case["Hkv"] if nq else 0):
            k = _exact_rows(s["cache"][0], s["cache"][1], slots, h, s["bits"])
            x = s["q"][rows, h * G:(h + 1) * G].double() * s["scale"]
            sc = (x.flatten(0, 1) @ k.T.contiguous()).view(nq, G, n)
            if case["causal"]:
                sc = torch.where(torch.tril(torch.ones(nq, n, dtype=torch.bool, device="cuda"), n - nq)[:, None, :], sc, -math.inf)
            yield b, h, slots, rows, sc


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "evict":
        return _exact_evict(case, s)
    H, Hkv = case["H"], case["Hkv"]
    G = H // Hkv
    if case["kind"] == "chunk":
        T = s["q"].shape[0]
        o, lse = torch.zeros(T, H, case["dv"], dtype=torch.float64, device="cuda"), torch.zeros(H, T, dtype=torch.float64, device="cuda")
        for _, h, slots, rows, sc in _exact_attention(case, s):
            mine = torch.arange(h * G, (h + 1) * G, device="cuda")
            if len(slots) == 0:
                lse[mine[:, None], rows] = -math.inf
                continue
            lse[mine[:, None], rows] = torch.logsumexp(sc, -1).T
            v = _exact_rows(s["cache"][2], s["cache"][3], slots, h, s["bits"])
            o[rows[:, None], mine] = (torch.softmax(sc, -1).flatten(0, 1) @ v).view(len(rows), G, -1)
        return o, lse
    w = s["weights"].double()
    page = case["page"]
    for _, h, slots, rows, sc in _exact_attention(case, s):
        sums = torch.exp(sc - s["lse_rows"][rows, h * G:(h + 1) * G].double()[..., None]).sum((0, 1))
        old = w[slots // page, h, slots % page]
        if s["fresh"]:
            old[len(slots) - len(rows):] = 0.0
        w[slots // page, h, slots % page] = old + sums
    return w


def _exact_evict(case, s):
    """Row by row on the host."""
    whole = [t.cpu().numpy().copy() for t in (s["weights"], *s["cache"])]
    w, table, page = whole[0], s["table"].cpu().numpy(), case["page"]
    left = []
    for b, n in enumerate(_lengths(case)[1]):
        keep = case["keep"]
        left.append(min(n, keep))
        if n <= keep:
            continue
        recent = min(case["recent"], keep)
        stay = keep - recent
        for h in range(case["Hkv"]):
            j = np.arange(n)
            p, at = table[b, j // page], j % page
            best = np.lexsort((j[:n - recent], -w[p, h, at][:n - recent]))[:stay]
            stays = np.zeros(n, dtype=bool)
            stays[best] = True
            to = np.concatenate((np.flatnonzero(~stays[:stay]), np.arange(stay, keep)))
            of = np.concatenate((stay + np.flatnonzero(stays[stay:]), np.arange(n - recent, n)))
            for t in whole:
                t[p[to], h, at[to]] = t[p[of], h, at[of]]
    w = torch.from_numpy(w.astype(np.float64)).cuda()
    return (torch.tensor(left, dtype=torch.int32, device="cuda"), w, *(torch.from_numpy(t).cuda() for t in whole[1:]))
