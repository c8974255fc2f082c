"""GPU tests of attn_cache_weigh against the definition in 64 bits (tolerances: cache_reference.weigh)."""
import math

import pytest
import torch

import cache_reference as cref
from cache_reference import BF, DIMS, HF
from test_gpu_cache_chunk import MIX, _case

pytestmark = pytest.mark.gpu


def _check(q, lse, before, after, cache, t, cu, lens, scale, causal, fresh, bits):
    """Everything on the CPU; lse [H, T]."""
    page = cache[0].shape[2]
    touched = torch.zeros_like(before, dtype=torch.bool)
    for b in range(len(lens)):
        i0, i1 = int(cu[b]), int(cu[b + 1])
        n = min(max(int(lens[b]), 0), t.shape[1] * page)
        if i1 <= i0 or n == 0:
            continue
        j = torch.arange(n)
        p, at = t[b, j // page].long(), j % page
        there = (p >= 0) & (p < cache[0].shape[0])
        k = torch.zeros(n, cache[0].shape[1], cache[1].shape[3] * 32, dtype=torch.float64)
        k[there] = cref.ref.rows(cache[0], cache[1], (p * page + at)[there], bits)
        got, off = cref.weigh(q[i0:i1].double(), lse[:, i0:i1], k, scale, causal)
        old = before[p * there, :, at].double()
        new = (j >= n - (i1 - i0))[:, None] & torch.tensor(fresh)
        want = torch.where(new, 0.0, old) + got
        diff = (after[p * there, :, at].double() - want).abs()
        assert (diff <= off + cref.STEP * want.abs())[there].all(), f"sequence {b}: {float((diff - off)[there].max())}"
        touched[p[there], :, at[there]] = True
    assert torch.equal(after[~touched], before[~touched])


def _lse(q, cache, t, cu, lens, scale, causal, bits):
    """The call's log-sum-exps, as fp32; rows of no sequence NaN."""
    out = torch.full((q.shape[1], q.shape[0]), math.nan)
    for b in range(len(lens)):
        i0, i1 = int(cu[b]), int(cu[b + 1])
        if i1 > i0:
            k, v = cref.rows(cache, t, b, max(int(lens[b]), 0), bits)
            out[:, i0:i1] = cref.attend(q[i0:i1].double(), k, v[..., :1], scale, causal)[1].float()
    return out


def _weights(g, cache):
    return torch.exp(2 * torch.randn(cache[0].shape[:3], generator=g))


@pytest.mark.parametrize("causal,fresh", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", DIMS)
def test_mixed_batch(dqk, dv, bits, causal, fresh):
    import paper_2603_05451_amd as A
    dtype = HF if bits == 8 else BF
    q, cache, t, cu, lens = _case(dqk + bits, MIX, 2, 3, dqk, dv, bits, 16, dtype)
    scale = dqk ** -0.5
    lse = _lse(q, cache, t, cu, lens, scale, causal, bits)
    w = _weights(cref.gen(1), cache)
    got = w.cuda()
    assert A.attn_cache_weigh(q.cuda(), lse.cuda(), got, cref.on_gpu(cache), t.cuda(), lens.cuda(), scale, causal, cu_seqlens=cu.cuda(), fresh=fresh) is got
    _check(q, lse, w, got.cpu(), cache, t, cu, lens, scale, causal, fresh, bits)


@pytest.mark.parametrize("Nq,G,page", [(1, 4, 64), (3, 8, 16), (40, 1, 128)])
def test_equal_batch(Nq, G, page):
    """The layout of attn_cache_fwd, views of q, and its own lse; an empty slot; every query's weights add up to one per head."""
    import paper_2603_05451_amd as A
    B, Hkv = 5, 2
    q, cache, t, cu, lens = _case(7, [(Nq, n) for n in (900, 64, 0, 65, 333)], Hkv, G, 128, 128, 4, page, BF)
    c = cref.on_gpu(cache)
    H = Hkv * G
    q4 = torch.zeros(B, H + 1, Nq, 128, dtype=BF, device="cuda").transpose(1, 2)[:, :, :H]
    q4.copy_(q.view(B, Nq, H, 128))
    _, lse = A.attn_cache_fwd(q4, c, t.cuda(), lens.cuda(), 0.09, True)
    w = _weights(cref.gen(2), cache)
    got = w.cuda()
    A.attn_cache_weigh(q4, lse, got, c, t.cuda(), lens.cuda(), 0.09, True)
    _check(q, lse.cpu().transpose(0, 1).reshape(H, B * Nq), w, got.cpu(), cache, t, cu, lens, 0.09, True, False, 4)
    zero = A.attn_cache_weights(c)
    A.attn_cache_weigh(q4, lse, zero, c, t.cuda(), lens.cuda(), 0.09, True)
    for b, n in enumerate(lens.tolist()):
        j = torch.arange(n)
        sums = zero.cpu()[t[b, j // page].long(), :, j % page].double().sum(0)
        assert (sums - min(n, Nq) * G).abs().max() < 1e-4 * Nq * G


def test_long_chunk():
    """Keys of several groups, rows of many tiles."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(3, [(500, 1900), (0, 5), (333, 700)], 1, 4, 128, 128, 4, 64, BF)
    c = cref.on_gpu(cache)
    _, lse = A.attn_cache_chunk_fwd(q.cuda(), c, t.cuda(), cu.cuda(), lens.cuda(), 0.09, True)
    w = _weights(cref.gen(3), cache)
    got = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse, got, c, t.cuda(), lens.cuda(), 0.09, True, cu_seqlens=cu.cuda(), fresh=True)
    _check(q, lse.cpu(), w, got.cpu(), cache, t, cu, lens, 0.09, True, True, 4)
    again = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse, again, c, t.cuda(), lens.cuda(), 0.09, True, cu_seqlens=cu.cuda(), fresh=True)
    assert torch.equal(got, again)


def test_many_sequences_and_bad_pages():
    import paper_2603_05451_amd as A
    g = cref.gen(5)
    seqs = [(int(a), int(n)) for a, n in zip(torch.randint(0, 6, (140,), generator=g), torch.randint(1, 90, (140,), generator=g))]
    q, cache, t, cu, lens = _case(6, seqs, 2, 2, 64, 64, 8, 16, BF)
    lse = _lse(q, cache, t, cu, lens, 0.125, False, 8)
    t[3, 0], t[77, 0], t[100, 0] = -1, cache[0].shape[0], 2 ** 31 - 1
    lens[9] = -4
    w = _weights(g, cache)
    got = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse.cuda(), got, cref.on_gpu(cache), t.cuda(), lens.cuda(), 0.125, False, cu_seqlens=cu.cuda())
    _check(q, lse, w, got.cpu(), cache, t, cu, lens, 0.125, False, False, 8)


def test_keys_that_are_not_finite():
    """A NaN key has the weight NaN, and no other key has (with the lse of the queries that do not see it)."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(8, [(70, 70)], 2, 1, 64, 64, 4, 16, BF)
    lse = _lse(q, cache, t, cu, lens, 0.125, True, 4)
    p, at = int(t[0, 40 // 16]), 40 % 16
    cache[1][p, 1, at] = 255
    for j in range(70, 80):                                    # behind the last key
        for x in cache:
            x[int(t[0, 4]), :, j % 16] = 255
    w = torch.ones(cache[0].shape[:3])
    got = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse.cuda(), got, cref.on_gpu(cache), t.cuda(), lens.cuda(), 0.125, True, cu_seqlens=cu.cuda())
    got = got.cpu()
    assert torch.isnan(got[p, 1, at]) and int(torch.isnan(got).sum()) == 1


def test_stream_and_graph():
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = (x.cuda() if torch.is_tensor(x) else x for x in _case(4, [(1, 300), (20, 90), (1, 10)], 2, 2, 128, 128, 4, 16, BF))
    c = cref.on_gpu(cache)
    _, lse = A.attn_cache_chunk_fwd(q, c, t, cu, lens, 0.1, True)
    start = _weights(cref.gen(1), cache).cuda()
    w = start.clone()
    call = lambda **kw: A.attn_cache_weigh(q, lse, w, c, t, lens, 0.1, True, cu_seqlens=cu, fresh=True, **kw)
    call()
    want, = w.clone(),
    w.copy_(start)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(stream=side)
    side.synchronize()
    assert torch.equal(w, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        w.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, want)
