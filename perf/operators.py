"""The operators on both sides of the attention calls, and the cases that their speed and results are followed on.

  rope       attn_rope_fwd           head norms (optional) and rotary positions of q and k in one pass
  rope_bwd   attn_rope_bwd           its gradients, those of the norms' weights among them
  store      attn_cache_write, then attn_cache_read of what was written: a paged cache quantised as it is written
  load       attn_cache_read         rows of a quantised cache back in 16 bits, as a prompt chunk's attention wants them
  attend     attn_cache_fwd          attention of few queries per sequence over a paged cache held in 4 or 8 bits

Where `own` is false the same is computed in elementary torch operations in 32 bits (angles and the sums over all rows in 64).

A quantised row (token, KV head) is in blocks of 32 channels, each with one scale byte s for 2^(s - 127).  4 bits: e2m1 codes, two to
a byte, the even channel in the low half; 8 bits: e4m3 codes.  The scale is the smallest with which no element of the block saturates
when it is rounded to nearest, ties to even.
"""
import math

import torch

own = False

NEVER = -1                                      # slot of a row that is padding: not written, read as zeros
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _rope(name, kind, B, N, H, Hkv, d, rot, offset=0, inter=False, norm=False, dtype="bf16", layout="dense", far=0):
    return {"name": name, "kind": kind, "B": B, "N": N, "H": H, "Hkv": Hkv, "d": d, "rot": rot, "offset": offset,
            "inter": inter, "norm": norm, "dtype": dtype, "layout": layout, "far": far}


def _store(name, T, Hkv, dqk, dv, bits, page, pages, dtype="bf16", pad=0):
    return {"name": name, "kind": "store", "T": T, "Hkv": Hkv, "dqk": dqk, "dv": dv, "bits": bits, "page": page, "pages": pages,
            "dtype": dtype, "pad": pad}


def _load(name, T, Hkv, dqk, dv, bits, page, pages, dtype="bf16"):
    return {"name": name, "kind": "load", "T": T, "Hkv": Hkv, "dqk": dqk, "dv": dv, "bits": bits, "page": page, "pages": pages,
            "dtype": dtype}


def _attend(name, B, Nq, H, Hkv, dqk, dv, bits, page, lo, hi, len_seed=0, causal=True, dtype="bf16", empty=0):
    return {"name": name, "kind": "attend", "B": B, "Nq": Nq, "H": H, "Hkv": Hkv, "dqk": dqk, "dv": dv, "bits": bits, "page": page,
            "lo": lo, "hi": hi, "len_seed": len_seed, "causal": causal, "dtype": dtype, "empty": empty}


def listed():
    return [
        # q and k of one decode step of 32 requests of a grouped-query model with head norms: latency
        _rope("rope_decode_B32", "rope", 32, 1, 32, 8, 128, 128, norm=True, far=131072),
        # a prompt of the same heads, rotation alone
        _rope("rope_prompt_N8192", "rope", 2, 8192, 32, 8, 128, 128, far=0),
        # fp16 encoder: slices of a fused projection, norms, half of the head rotated in neighbouring pairs, odd length
        _rope("rope_norm_qkv_d64_fp16_N1000", "rope", 8, 1000, 12, 12, 64, 32, inter=True, norm=True, dtype="fp16", layout="qkv"),
        # backward of norms and rotation in the benchmark's training step
        _rope("rope_bwd_norm_N8192", "rope_bwd", 2, 8192, 16, 16, 128, 128, norm=True),
        # backward of latent-attention heads, of which the last 64 dims carry the position
        _rope("rope_bwd_d192_tail_N4096", "rope_bwd", 1, 4096, 16, 16, 192, 64, offset=128, far=4096),
        # new tokens of one decode step into the cache, empty batch slots among them, and back
        _store("store_decode_B48", 48, 8, 128, 128, 4, 64, 1024, pad=5),
        # a prompt chunk into a cache of 8 bits, and back for the chunk's own attention
        _store("store_prompt_T8192_8bit", 8192, 8, 128, 128, 8, 16, 2048),
        # the cache of one long request read back for a chunk against it
        _load("load_T30001", 30001, 8, 128, 128, 4, 64, 1024),
        # one token of one request against a long context
        _attend("attend_B1_N32000", 1, 1, 32, 8, 128, 128, 4, 64, 32000, 32000),
        # one decode step of 32 requests of equal lengths
        _attend("attend_B32_N4001", 32, 1, 32, 8, 128, 128, 4, 16, 4001, 4001),
        # one decode step of a serving batch whose requests are at different lengths, four slots empty
        _attend("attend_mixed_B48", 48, 1, 32, 8, 128, 128, 4, 64, 64, 8192, len_seed=12, empty=4),
        # four drafted tokens per request, fp16, small heads, 8 bits
        _attend("attend_draft4_d64_8bit_fp16", 16, 4, 16, 4, 64, 64, 8, 32, 100, 2000, len_seed=3, dtype="fp16"),
    ]


DIMS = [(64, 64), (96, 96), (128, 128), (192, 128), (256, 256)]


def draw(rng):
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        kind = rng.choice(["rope", "rope", "rope_bwd", "rope_bwd", "store", "store", "load", "attend", "attend", "attend"])
        dtype = "fp16" if rng.random() < 0.3 else "bf16"
        Hkv = rng.choice([1, 2, 4, 8, 8, 16])
        H = Hkv * rng.choice([1, 2, 4, 4, 8])
        dqk, dv = rng.choice(DIMS + [(128, 128), (128, 128)])
        if H > 64:
            continue
        if kind in ("rope", "rope_bwd"):
            rot = 16 * rng.randint(1, dqk // 16) if rng.random() < 0.4 else dqk
            offset = 8 * rng.randint(0, (dqk - rot) // 8)
            c = _rope("", kind, logu(1, 32), logu(1, 8192), H, Hkv, dqk, rot, offset, rng.random() < 0.4, rng.random() < 0.6, dtype,
                      rng.choice(["dense", "qkv", "bhnd"]), rng.choice([0, 0, 4096, 1 << 20]))
        elif kind == "store":
            T, page = logu(1, 16384), 1 << rng.randint(4, 8)
            c = _store("", T, Hkv, dqk, dv, rng.choice([4, 4, 8]), page, (T + page - 1) // page + rng.randint(1, 64), dtype,
                       rng.randint(0, T // 8))
        elif kind == "load":
            T, page = logu(1, 65536), 1 << rng.randint(4, 8)
            c = _load("", T, Hkv, dqk, dv, rng.choice([4, 4, 8]), page, (T + page - 1) // page + rng.randint(1, 64), dtype)
        else:
            B, hi = logu(1, 128), logu(16, 32768)
            lo = hi if rng.random() < 0.3 else max(1, hi // rng.choice([2, 8, 64]))
            c = _attend("", B, rng.choice([1, 1, 1, 2, 3, 4, 8]), H, Hkv, dqk, dv, rng.choice([4, 4, 8]), 1 << rng.randint(4, 8),
                        lo, hi, rng.randrange(1 << 20), rng.random() < 0.8, dtype, rng.randint(0, B // 4) if B > 3 else 0)
            if c["B"] * c["hi"] * c["Hkv"] * c["dqk"] > 600e6:          # the plain form holds every sequence at the longest length
                continue
        if work(c)["bytes"] <= 3.2e8:
            del c["name"]
            return c


def _lengths(case):
    """Key lengths of an attend case: log-uniform in [lo, hi], some slots of the batch empty."""
    import random
    r = random.Random(case["len_seed"])
    lens = [int(round(math.exp(r.uniform(math.log(case["lo"]), math.log(case["hi"]))))) for _ in range(case["B"])]
    for i in r.sample(range(case["B"]), case["empty"]):
        lens[i] = 0
    return lens


def work(case):
    kind = case["kind"]
    if kind in ("rope", "rope_bwd"):
        row = case["B"] * case["N"] * (case["H"] + case["Hkv"]) * case["d"]
        if kind == "rope":
            return {"bytes": 2 * row * 2, "flops": row * (7 if case["norm"] else 3)}
        return {"bytes": 2 * row * (3 if case["norm"] else 2), "flops": row * (15 if case["norm"] else 3)}
    if kind in ("store", "load"):
        n = case["T"] * case["Hkv"] * (case["dqk"] + case["dv"])
        code = n * case["bits"] // 8 + n // 32
        return {"bytes": n * 2 * 2 + code * 2 if kind == "store" else n * 2 + code, "flops": 4 * n if kind == "store" else n}
    lens, Nq, H, Hkv, d2 = _lengths(case), case["Nq"], case["H"], case["Hkv"], case["dqk"] + case["dv"]
    n = sum(lens) * Hkv * d2
    pairs = sum(sum(max(0, min(L, L - Nq + i + 1)) for i in range(Nq)) if case["causal"] else L * Nq for L in lens)
    return {"bytes": n * case["bits"] // 8 + n // 32 + case["B"] * Nq * H * (2 * d2 + 4), "flops": 2 * pairs * H * d2}


# ---------------------------------------------------------------------------------------------------------------------------
# the plain forms

def _freqs(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()


def _angles(s):
    """cos and sin [B, N, 1, rot / 2] of position * frequency, the angle in 64 bits."""
    a = s["positions"].double()[:, :, None, None] * s["freqs"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _turn(x, s, c, sn):
    """The rotation of the pairs of x, in 32 bits; the other dims as they are."""
    lo, hi = s["offset"], s["offset"] + 2 * s["freqs"].numel()
    part = x[..., lo:hi]
    if s["inter"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((a * c - b * sn, a * sn + b * c), dim=-1).flatten(-2)
    else:
        a, b = part.chunk(2, dim=-1)
        turned = torch.cat((a * c - b * sn, a * sn + b * c), dim=-1)
    return torch.cat((x[..., :lo], turned, x[..., hi:]), dim=-1)


def _plain_rope(x, w, s, c, sn):
    y = x.float()
    if s["eps"] is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * w.float()
    return _turn(y, s, c, sn).to(x.dtype)


def _plain_rope_bwd(dy, x, w, s, c, sn):
    g = _turn(dy.float(), s, c, -sn)
    if s["eps"] is None:
        return g.to(dy.dtype), None
    xf = x.float()
    r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + s["eps"])
    dw = (g * xf * r).sum(dim=(0, 1, 2), dtype=torch.float64).float()
    g = g * w.float()
    return (r * (g - xf * r * r * (g * xf).mean(-1, keepdim=True))).to(dy.dtype), dw


def _round_blocks(x, bits):
    """What the cache holds for x [..., d]: (codes as integers, scale bytes as integers), blocks of 32 along the last axis."""
    b = x.float().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)                                     # amax = m 2^e, 1/2 <= m < 1
    if bits == 4:
        e = torch.where(8.0 * m < 7.0, e - 3, e - 2)
    else:
        e = torch.where(512.0 * m <= 464.0, e - 9, e - 8)
    e = torch.where(amax == 0, -127, e).clamp(min=-127)
    bad = ~torch.isfinite(amax)
    y = torch.where(bad, 0.0, torch.ldexp(torch.ldexp(b, -(e // 2)), e // 2 - e))
    a = y.abs()
    if bits == 4:
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        v = torch.round(a / step) * step                         # half to even, as are the codes
        code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).int()
        code = code + 8 * torch.signbit(y).int()
    else:
        ex = (torch.frexp(a)[1] - 1).clamp(min=-6)
        n = torch.round(torch.ldexp(a, 3 - ex))                  # multiples of 2^(ex - 3): 8 .. 16, below 8 where subnormal
        code = n.int() + 8 * (ex + 6) + 128 * torch.signbit(y).int()
    return code.flatten(-2), torch.where(bad, 255, e + 127).squeeze(-1)


def _values(code, scale, bits):
    """The numbers, in 32 bits, that codes [..., d] with scale bytes [..., d / 32] stand for."""
    code, scale = code.int(), scale.int()
    if bits == 4:
        v = torch.tensor(_E2M1, device=code.device)[(code & 7).long()]
        neg = code & 8
    else:
        ex, man = (code >> 3) & 15, (code & 7).float()
        v = torch.ldexp(torch.where(ex == 0, man, man + 8.0), ex.clamp(min=1) - 10)
        neg = code & 128
    v = torch.where(neg != 0, -v, v).unflatten(-1, (-1, 32))
    e = (scale - 127)[..., None]
    v = torch.ldexp(torch.ldexp(v, e // 2), e - e // 2)
    return torch.where((scale == 255)[..., None], math.nan, v).flatten(-2)


def _unpacked(bytes_, bits):
    return bytes_ if bits == 8 else torch.stack((bytes_ & 15, bytes_ >> 4), dim=-1).flatten(-2)


def _packed(code, bits):
    code = code.to(torch.uint8)
    return code if bits == 8 else code[..., 0::2] | (code[..., 1::2] << 4)


def _cached(codes, scales, slots, bits):
    """Rows [..., Hkv, d] in 32 bits of the cache at slots [...]."""
    page = codes.shape[2]
    p, at = slots // page, slots % page
    return _values(_unpacked(codes[p, :, at], bits), scales[p, :, at], bits)


def _plain_attend(s):
    q, (kc, ks, vc, vs), lens = s["q"], s["cache"], s["lens"].long()
    B, Nq, H, dqk = q.shape
    Hkv, page, bits, longest = kc.shape[1], kc.shape[2], s["bits"], s["longest"]
    j = torch.arange(longest, device=q.device)
    slots = s["table"].long()[:, j // page] * page + j % page                          # [B, M]
    k = _cached(kc, ks, slots, bits).transpose(1, 2)                                    # [B, Hkv, M, d]
    v = _cached(vc, vs, slots, bits).transpose(1, 2)
    G = H // Hkv
    qg = q.float().reshape(B, Nq, Hkv, G, dqk).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Nq * G, dqk)
    sc = torch.matmul(qg, k.transpose(2, 3).contiguous()).mul_(s["scale"]).view(B, Hkv, Nq, G, longest)
    last = lens[:, None] - 1 - (torch.arange(Nq - 1, -1, -1, device=q.device) if s["causal"] else torch.zeros(Nq, device=q.device).long())
    hidden = (j > last[:, :, None])[:, None, :, None, :]                                # [B, 1, Nq, 1, M]
    sc = sc.masked_fill(hidden, -math.inf)
    m = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(sc - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, Nq * G, longest), v.contiguous()).view(B, Hkv, Nq, G, -1)
    o = torch.where(l > 0, o / l, 0.0)
    lse = torch.where(l > 0, m + torch.log(l), -math.inf)[..., 0]
    return (o.permute(0, 2, 1, 3, 4).reshape(B, Nq, H, -1).to(q.dtype), lse.permute(0, 1, 3, 2).reshape(B, H, Nq))


# ---------------------------------------------------------------------------------------------------------------------------

def _some_cache(case, normal, gen):
    """A cache whose every slot holds values as a model's keys and values have them (N(0, 1), a few channels eight times that)."""
    pages, Hkv, page, bits = case["pages"], case["Hkv"], case["page"], case["bits"]
    out = []
    for d in (case["dqk"], case["dv"]):
        codes = torch.empty(pages, Hkv, page, d * bits // 8, dtype=torch.uint8, device="cuda")
        scales = torch.empty(pages, Hkv, page, d // 32, dtype=torch.uint8, device="cuda")
        outliers = torch.where(torch.rand(Hkv, 1, d, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
        step = max(1, (1 << 24) // (Hkv * page * d))
        for i in range(0, pages, step):
            n = min(step, pages - i)
            c, e = _round_blocks(normal(n, Hkv, page, d) * outliers, bits)
            codes[i:i + n], scales[i:i + n] = _packed(c, bits), e.to(torch.uint8)
        out += [codes, scales]
    return tuple(out)


def prepare(case, seed):
    dtype = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, dtype=torch.float32, device="cuda")
    kind = case["kind"]
    s = {"kind": kind}
    if kind in ("rope", "rope_bwd"):
        B, N, H, Hkv, d = (case[n] for n in ("B", "N", "H", "Hkv", "d"))

        def pair():
            if case["layout"] == "qkv":
                qkv = normal(B, N, H + 2 * Hkv, d).to(dtype)
                return qkv[:, :, :H], qkv[:, :, H:H + Hkv]
            if case["layout"] == "bhnd":
                return tuple(normal(B, h, N, d).to(dtype).transpose(1, 2) for h in (H, Hkv))
            return tuple(normal(B, N, h, d).to(dtype) for h in (H, Hkv))

        s["q"], s["k"] = pair()
        if kind == "rope_bwd":
            s["dq"], s["dk"] = pair()
        s["freqs"] = _freqs(case["rot"]).cuda()
        start = torch.randint(0, case["far"] + 1, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
        s["positions"] = start + torch.arange(N, device="cuda", dtype=torch.int32)
        s["offset"], s["inter"], s["eps"] = case["offset"], case["inter"], 1e-6 if case["norm"] else None
        s["wq"], s["wk"] = ((1 + 0.2 * normal(d)).to(dtype) for _ in range(2)) if case["norm"] else (None, None)
        return s
    s["bits"] = case["bits"]
    if kind == "attend":
        B, Nq, H, dqk, page = case["B"], case["Nq"], case["H"], case["dqk"], case["page"]
        lens = _lengths(case)
        need = [(n + page - 1) // page for n in lens]
        case = dict(case, pages=max(1, sum(need)))
        s["longest"] = max(1, max(lens))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["q"] = normal(B, Nq, H, dqk).to(dtype)
        order = torch.randperm(case["pages"], generator=gen, device="cuda").int()       # pages as a server hands them out
        width = max(1, max(need))
        at = torch.tensor([sum(need[:b]) for b in range(B)], device="cuda")[:, None] + torch.arange(width, device="cuda")
        held = torch.arange(width, device="cuda") < torch.tensor(need, device="cuda")[:, None]
        s["table"] = torch.where(held, order[at.clamp(max=case["pages"] - 1)], 0).int().contiguous()
        s["scale"], s["causal"] = dqk ** -0.5, case["causal"]
    else:
        T, total = case["T"], case["pages"] * case["page"]
        s["slots"] = torch.randperm(total, generator=gen, device="cuda")[:T].int()
        if kind == "load":                                       # a request's pages lie anywhere, its rows in order inside them
            page = case["page"]
            order = torch.randperm(case["pages"], generator=gen, device="cuda").int()
            t = torch.arange(T, device="cuda")
            s["slots"] = (order[t // page] * page + t % page).int()
        elif case["pad"]:
            s["slots"][torch.randperm(T, generator=gen, device="cuda")[:case["pad"]]] = NEVER
        if kind == "store":
            s["k"], s["v"] = (normal(T, case["Hkv"], d).to(dtype) for d in (case["dqk"], case["dv"]))
        s["dtype"] = dtype
    s["cache"] = _some_cache(case, normal, gen)
    return s


def run(s):
    kind = s["kind"]
    if own:
        import paper_2603_05451_amd as A
        if kind == "rope":
            return A.attn_rope_fwd(s["q"], s["k"], s["freqs"], s["positions"], interleaved=s["inter"], offset=s["offset"], eps=s["eps"],
                                   q_weight=s["wq"], k_weight=s["wk"])
        if kind == "rope_bwd":
            norm = s["eps"] is not None
            out = A.attn_rope_bwd(s["dq"], s["dk"], s["freqs"], s["positions"], interleaved=s["inter"], offset=s["offset"], eps=s["eps"],
                                  q=s["q"] if norm else None, k=s["k"] if norm else None, q_weight=s["wq"], k_weight=s["wk"])
            return out if norm else out[:2]
        cache = A.AttnCache(*s["cache"])
        if kind == "store":
            A.attn_cache_write(s["k"], s["v"], s["slots"], cache)
            return A.attn_cache_read(s["slots"], cache, s["dtype"])
        if kind == "load":
            return A.attn_cache_read(s["slots"], cache, s["dtype"])
        return A.attn_cache_fwd(s["q"], cache, s["table"], s["lens"], s["scale"], s["causal"])
    if kind in ("rope", "rope_bwd"):
        c, sn = _angles(s)
        if kind == "rope":
            return _plain_rope(s["q"], s["wq"], s, c, sn), _plain_rope(s["k"], s["wk"], s, c, sn)
        dq, dwq = _plain_rope_bwd(s["dq"], s["q"], s["wq"], s, c, sn)
        dk, dwk = _plain_rope_bwd(s["dk"], s["k"], s["wk"], s, c, sn)
        return (dq, dk) if dwq is None else (dq, dk, dwq, dwk)
    if kind == "attend":
        return _plain_attend(s)
    there = (s["slots"] >= 0)[:, None, None]
    if kind == "store":
        return tuple(torch.where(there, _values(*_round_blocks(x, s["bits"]), s["bits"]), 0.0).to(s["dtype"]) for x in (s["k"], s["v"]))
    kc, ks, vc, vs = s["cache"]
    at = s["slots"].long().clamp(min=0)
    return tuple(torch.where(there, _cached(c, e, at, s["bits"]), 0.0).to(s["dtype"]) for c, e in ((kc, ks), (vc, vs)))


# ---------------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_pairs(s, d):
    """Index of the first and second dim of every rotated pair."""
    n = s["freqs"].numel()
    i = torch.arange(n, device="cuda")
    return (s["offset"] + 2 * i, s["offset"] + 2 * i + 1) if s["inter"] else (s["offset"] + i, s["offset"] + n + i)


def _exact_rope(s, name, weight, grad=None):
    x = s[name].double()
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                    s["positions"].double()[:, :, None, None] * s["freqs"].double())
    i, j = _exact_pairs(s, x.shape[-1])
    norm = s["eps"] is not None
    inv = (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).pow(-0.5) if norm else None
    if grad is None:
        y = x * inv * weight.double() if norm else x.clone()
        t = torch.complex(y[..., i], y[..., j]) * z
        y[..., i], y[..., j] = t.real, t.imag
        return y
    g = s[grad].double()
    t = torch.complex(g[..., i], g[..., j]) * z.conj()
    g = g.clone()
    g[..., i], g[..., j] = t.real, t.imag
    if not norm:
        return g
    hat = x * inv
    dhat = g * weight.double()
    return inv * (dhat - hat * (dhat * hat).sum(-1, keepdim=True) / x.shape[-1]), (g * hat).flatten(0, 2).sum(0)


def _grid(bits):
    """The non-negative numbers of the code, in order: index parity is the parity of the mantissa's last bit."""
    if bits == 4:
        return torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    return torch.tensor([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64, device="cuda")


def _exact_store(x, bits):
    grid = _grid(bits)
    top = 7.0 if bits == 4 else 464.0
    b = x.double().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / top)).clamp(min=-127)       # the least with amax <= top 2^e, up to the logarithm's rounding
    fits = lambda e: (amax < top * 2.0 ** e) if bits == 4 else (amax <= top * 2.0 ** e)
    e = torch.where(fits(e - 1) & (e > -127), e - 1, e)
    e = torch.where(fits(e), e, e + 1)
    a = b.abs() / 2.0 ** e
    hi = torch.searchsorted(grid, a.contiguous()).clamp(1, len(grid) - 1)
    lo = hi - 1
    up = (grid[hi] - a < a - grid[lo]) | ((grid[hi] - a == a - grid[lo]) & (hi % 2 == 0))
    return (torch.where(up, grid[hi], grid[lo]) * torch.sign(b) * 2.0 ** e).flatten(-2)


def _exact_rows(codes, scales, slots, bits):
    page = codes.shape[2]
    grid = _grid(bits)
    half = len(grid) if bits == 4 else 128
    table = torch.cat((grid, torch.full((half - len(grid),), math.nan, dtype=torch.float64, device="cuda")))
    table = torch.cat((table, -table))
    raw = codes[slots // page, :, slots % page]
    code = raw.long() if bits == 8 else torch.stack((raw.long() % 16, raw.long() // 16), -1).flatten(-2)
    return table[code] * (2.0 ** (scales[slots // page, :, slots % page].double() - 127)).repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return _exact_rope(s, "q", s["wq"]), _exact_rope(s, "k", s["wk"])
    if kind == "rope_bwd":
        q, k = _exact_rope(s, "q", s["wq"], "dq"), _exact_rope(s, "k", s["wk"], "dk")
        return (q[0], k[0], q[1], k[1]) if case["norm"] else (q, k)
    bits = case["bits"]
    kc, ks, vc, vs = s["cache"]
    if kind == "store":
        there = (s["slots"] >= 0)[:, None, None]
        return tuple(_exact_store(x, bits) * there for x in (s["k"], s["v"]))
    if kind == "load":
        return tuple(_exact_rows(c, e, s["slots"].long(), bits) for c, e in ((kc, ks), (vc, vs)))
    q, table = s["q"], s["table"].long()
    B, Nq, H, _ = q.shape
    Hkv, page = kc.shape[1], kc.shape[2]
    o = torch.zeros(B, Nq, H, case["dv"], dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, Nq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        j = torch.arange(n, device="cuda")
        slots = table[b, j // page] * page + j % page
        k, v = (_exact_rows(c, e, slots, bits).repeat_interleave(H // Hkv, 1) for c, e in ((kc, ks), (vc, vs)))
        for i in range(Nq):
            seen = n - Nq + i + 1 if case["causal"] else n
            if seen > 0:
                sc = (k[:seen] * q[b, i].double()).sum(-1) * s["scale"]                # [seen, H]
                lse[b, :, i] = torch.logsumexp(sc, 0)
                o[b, i] = (torch.softmax(sc, 0)[:, :, None] * v[:seen]).sum(0)
    return o, lse
