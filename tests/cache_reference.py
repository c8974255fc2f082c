"""Definitions in 64 bits, on the CPU, of attention of chunks over the quantised cache, of the weight that its keys had, and of eviction."""
import math

import torch

import ops_reference as ref

BF, HF = torch.bfloat16, torch.float16
DIMS = [(64, 64), (96, 96), (128, 128), (192, 128), (256, 256)]
STEP = 2.0 ** -24


def gen(seed):
    return torch.Generator("cpu").manual_seed(seed)


def random_cache(g, pages, page, Hkv, dqk, dv, bits):
    """A cache of random finite codes and scales about 1, on the CPU."""
    out = []
    for d in (dqk, dv):
        raw = torch.randint(0, 256, (pages, Hkv, page, d * bits // 8), generator=g, dtype=torch.uint8)
        if bits == 8:
            raw = torch.where((raw & 0x7f) > 0x47, raw & 0xb7, raw)
        out += [raw, torch.randint(123, 127, (pages, Hkv, page, d // 32), generator=g).to(torch.uint8) - (2 if bits == 8 else 0)]
    return out


def on_gpu(cache):
    import paper_2603_05451_amd as A
    return A.AttnCache(*(t.cuda() for t in cache))


def table(g, lens, page, pages, width=None):
    """Distinct pages for every sequence, in no order; nonsense behind the last one."""
    need = [max(0, -(-n // page)) for n in lens]
    width = width or max(1, max(need))
    order = torch.randperm(pages, generator=g)
    t = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(lens), width), generator=g).int()
    i = 0
    for b, n in enumerate(need):
        t[b, :n] = order[i:i + n]
        i += n
    return t


def rows(cache, t, b, n, bits):
    """Keys and values [n, Hkv, d] of sequence b in 64 bits."""
    page, j = cache[0].shape[2], torch.arange(n)
    slots = t[b, j // page].long() * page + j % page
    return tuple(ref.rows(cache[i], cache[i + 1], slots, bits) for i in (0, 2))


def limits(nq, n, causal):
    """The last key that each query sees."""
    return torch.arange(n - nq, n) if causal else torch.full((nq,), n - 1)


def scores(q, k, scale, causal):
    """q [nq, H, d], k [n, Hkv, d] -> (scores [H, nq, n], -inf where a key is not seen; the sizes of what they are sums of)."""
    nq, n, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    kk = k.repeat_interleave(G, 1).permute(1, 2, 0).contiguous()
    qq = q.transpose(0, 1).contiguous()
    hidden = torch.arange(n) > limits(nq, n, causal)[:, None]
    s, size = qq @ kk * scale, qq.abs() @ kk.abs() * scale
    return s.masked_fill(hidden, -math.inf), size.masked_fill(hidden, 0.0)


def attend(q, k, v, scale, causal):
    """-> (o [nq, H, dv], lse [H, nq], size of what o is the sum of, largest size of a score's terms [H, nq])."""
    nq, H, n = q.shape[0], q.shape[1], k.shape[0]
    if n == 0:
        z = torch.zeros(nq, H, v.shape[-1], dtype=torch.float64)
        return z, torch.full((H, nq), -math.inf, dtype=torch.float64), z, torch.zeros(H, nq, dtype=torch.float64)
    s, terms = scores(q, k, scale, causal)
    lse = torch.logsumexp(s, -1)
    p = torch.where(torch.isneginf(lse)[..., None], 0.0, torch.exp(s - lse[..., None]))
    vv = v.repeat_interleave(H // v.shape[1], 1).transpose(0, 1).contiguous()
    return (p @ vv).transpose(0, 1), lse, (p @ vv.abs()).transpose(0, 1), terms.amax(-1)


def check_attention(q, cache, t, cu, lens, scale, causal, o, lse, bits, sequences=None):
    """o [T, H, dv] and lse [H, T] of attn_cache_chunk_fwd against 64 bits; everything on the CPU.

    Per element: the output's rounding, half a step of the result; P's rounding to the element type, half a step of sum_j P_j |V_j|; and fp32: a
    score, a sum of d products, is off by at most (d + 8) 2^-24 of its terms' sizes, which is what P is off relatively (and again through the row
    sum).  The row sum adds n / 2 terms per lane and the accumulators n, with a rescaling for every 32 keys at most and a merge: n + n / 32 + 64
    steps of 2^-24.  LSE: the score's error, the row sum's, and 2^-23 of itself."""
    half, page = ref.HALF[q.dtype], cache[0].shape[2]
    for b in range(len(lens)) if sequences is None else sequences:
        i0, i1 = int(cu[b]), int(cu[b + 1])
        if i1 <= i0:
            continue
        n = min(max(int(lens[b]), 0), t.shape[1] * page)
        k, v = rows(cache, t, b, n, bits)
        wo, wl, size, terms = attend(q[i0:i1].double(), k, v, scale, causal)
        got_o, got_l = o[i0:i1].double(), lse[:, i0:i1].double()
        none = torch.isneginf(wl)
        assert torch.equal(torch.isneginf(got_l), none), f"sequence {b}"
        steps = ((q.shape[2] + 8) * terms + n + n / 32 + 64) * STEP
        off = (got_l - wl).abs().masked_fill(none, 0.0)
        assert (off <= steps + 2 * STEP * wl.abs().masked_fill(none, 0.0)).all(), f"lse of sequence {b}"
        steps = steps.T[..., None]
        bound = half * wo.abs() + ref.TINY[q.dtype] + (half + 2 * steps) * (size + wo.abs())
        assert ((got_o - wo).abs() <= bound).all(), f"o of sequence {b}: {float(((got_o - wo).abs() / (bound + 1e-300)).max())} of the bound"
        assert (got_o.transpose(0, 1)[none] == 0).all()


def weigh(q, lse, k, scale, causal):
    """q [nq, H, d], lse [H, nq], k [n, Hkv, d] -> (weights [n, Hkv], how far off fp32 may be).

    A term exp(s - lse): the score is off by (d + 8) 2^-24 of its terms' sizes, the exponent of 2, s log2 e - lse log2 e, rounded twice, by two steps of
    |s| + |lse|, exp2 by two; the sum of R rows over R / 32 per lane and 32 lanes, by R / 32 + 40 steps."""
    nq, H, d = q.shape
    Hkv, n = k.shape[1], k.shape[0]
    s, terms = scores(q, k, scale, causal)
    there = ~torch.isneginf(lse)[..., None]
    p = torch.where(there, torch.exp(s - lse.double()[..., None]), 0.0)
    size = torch.where(there & torch.isfinite(s), (d + 8) * terms + 4 * (s.abs() + lse.double().abs()[..., None]) + 4, 0.0)
    fold = lambda x: x.view(Hkv, H // Hkv, nq, n).sum((1, 2)).T
    return fold(p), (fold(p * size) + (nq * (H // Hkv) / 32 + 40) * fold(p)) * STEP


def places(w, n, keep, recent):
    """Where the rows of a sequence come from: w [n] fp32 -> (to, of): row of[i] goes to place to[i], all others stay."""
    if n <= max(keep, 0):
        return [], []
    left = max(keep, 0)
    recent = min(recent, left)
    stay = left - recent
    value = lambda j: math.inf if math.isnan(w[j]) else float(w[j])
    best = sorted(range(n - recent), key=lambda j: (not math.isnan(w[j]), -value(j), j))[:stay]
    stays = set(best)
    holes = [j for j in range(stay) if j not in stays]
    movers = [j for j in range(stay, n - recent) if j in stays]
    return holes + list(range(stay, left)), movers + list(range(n - recent, n))
