"""GPU tests of attn_cache_evict: every byte of the cache and every weight against the definition row by row (exact)."""
import math

import pytest
import torch

import cache_reference as cref
from cache_reference import DIMS

pytestmark = pytest.mark.gpu


def _want(w, cache, t, lens, keep, recent):
    """CPU copies of what the call leaves."""
    w, cache = w.clone(), [x.clone() for x in cache]
    page, Hkv = cache[0].shape[2], cache[0].shape[1]
    for b, n in enumerate(lens.tolist()):
        n = min(max(n, 0), t.shape[1] * page)
        j = torch.arange(n)
        p, at = t[b, j // page].long(), j % page
        for h in range(Hkv):
            to, of = cref.places(w[p, h, at].tolist(), n, int(keep[b]), recent)
            if to:
                for x in (w, *cache):
                    x[p[to], h, at[to]] = x[p[of], h, at[of]].clone()
    return w, cache


def _case(seed, lens, Hkv, dqk, dv, bits, page, spare=3, width=None):
    g = cref.gen(seed)
    pages = sum(-(-max(n, 0) // page) for n in lens) + spare
    cache = [torch.randint(0, 256, (pages, Hkv, page, c), generator=g, dtype=torch.uint8) for d in (dqk, dv) for c in (d * bits // 8, d // 32)]
    w = torch.exp(2 * torch.randn(pages, Hkv, page, generator=g))
    w = torch.where(torch.rand(w.shape, generator=g) < 0.3, torch.randint(0, 3, w.shape, generator=g).float(), w)         # many equal ones
    return cache, w, cref.table(g, lens, page, pages, width), torch.tensor(lens, dtype=torch.int32)


def _check(cache, w, t, lens, keep, recent, **kw):
    import paper_2603_05451_amd as A
    c, gw = cref.on_gpu(cache), w.cuda()
    keep = torch.tensor(keep, dtype=torch.int32)
    left = A.attn_cache_evict(gw, c, t.cuda(), lens.cuda(), keep.cuda(), recent, **kw)
    n = lens.clamp(min=0, max=t.shape[1] * cache[0].shape[2])
    assert left.dtype == torch.int32 and torch.equal(left.cpu(), torch.minimum(n, keep.clamp(min=0)))
    ww, wc = _want(w, cache, t, lens, keep, recent)
    assert torch.equal(gw.cpu().view(torch.int32), ww.view(torch.int32)), "weights"
    for x, y, name in zip(c, wc, c._fields):
        assert torch.equal(x.cpu(), y), name


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", DIMS)
def test_layouts(dqk, dv, bits):
    cache, w, t, lens = _case(dqk + bits, [100, 0, 33, 64, 1, 257], 3, dqk, dv, bits, 16)
    _check(cache, w, t, lens, [60, 5, 33, 10, 0, 100], 8)


@pytest.mark.parametrize("n,keep,recent", [(2, 1, 0), (2, 1, 1), (50, 49, 49), (50, 49, 0), (300, 299, 100), (300, 20, 20), (300, 20, 500), (300, 0, 3), (300, -1, 0),
                                           (4095, 4000, 7), (4097, 100, 99), (5000, 4096, 64), (9001, 3000, 0), (9001, 8990, 5000), (300, 299, 0)])
def test_sizes(n, keep, recent):
    """Lengths about the block's turns of 4096 keys; recent rows that overlap their new places."""
    cache, w, t, lens = _case(n + keep, [n, 17], 1, 64, 64, 4, 64)
    _check(cache, w, t, lens, [keep, 17], recent)


@pytest.mark.parametrize("kind", ["equal", "ascending", "descending", "special"])
def test_weights_in_order(kind):
    cache, w, t, lens = _case(1, [700], 2, 64, 64, 8, 32)
    j = torch.arange(700)
    p, at = t[0, j // 32].long(), j % 32
    for h in range(2):
        x = {"equal": torch.full((700,), 0.25), "ascending": j.float(), "descending": -j.float()}.get(kind)
        if x is None:
            x = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -3.4e38, -math.nan, 1.0])[torch.randint(0, 11, (700,), generator=cref.gen(h))]
        w[p, h, at] = x
    for keep, recent in ((100, 10), (350, 0), (650, 100), (699, 1)):
        _check(cache, w, t, lens, [keep], recent)


@pytest.mark.parametrize("of", [4096, 4097, 8191, 8192, 8193, 8197, 20001])
def test_ties_over_turns(of):
    """Rows that go are the last of those that are equal, zeros all over the sequence; turns of 4096 and of 8192 keys, and one more or less."""
    cache, w, t, lens = _case(of, [of + 5], 1, 64, 64, 4, 64)
    zeros = int((w[t[0, torch.arange(of) // 64].long(), 0, torch.arange(of) % 64] == 0).sum())
    _check(cache, w, t, lens, [of + 5 - zeros // 2], 5)


def test_long_sequence():
    cache, w, t, lens = _case(5, [70001], 1, 64, 64, 4, 256)
    _check(cache, w, t, lens, [20000], 300)
    _check(cache, w, t, lens, [69000], 300)


def test_many_sequences_wide_table():
    g = cref.gen(9)
    n = torch.randint(0, 200, (90,), generator=g).tolist()
    cache, w, t, lens = _case(2, n, 4, 128, 128, 4, 16, width=40)
    _check(cache, w, t, lens, torch.randint(0, 150, (90,), generator=g).tolist(), 16)


def test_lengths_beyond_the_table():
    cache, w, t, lens = _case(7, [96, 64], 2, 64, 64, 4, 32)
    lens[0], lens[1] = 2 ** 31 - 1, -7
    _check(cache, w, t, lens, [50, 5], 9)


def test_pages_outside_the_cache():
    """Their rows have the least weight; one that stays is NaN where it goes; nothing else changes."""
    import paper_2603_05451_amd as A
    cache, w, t, lens = _case(3, [80], 1, 64, 64, 4, 16)
    for bad in (-1, cache[0].shape[0], 2 ** 31 - 1):
        u = t.clone()
        u[0, 1] = bad                                                      # keys 16 ... 31
        c, gw = cref.on_gpu(cache), w.cuda()
        A.attn_cache_evict(gw, c, u.cuda(), lens.cuda(), torch.tensor([40], dtype=torch.int32).cuda(), 0)
        j = torch.arange(80)
        p, at = u[0, j // 16].long(), j % 16
        there = (p >= 0) & (p < cache[0].shape[0])
        x = torch.where(there, w[p * there, 0, at], -math.inf).tolist()
        to, of = cref.places(x, 80, 40, 0)
        ww, wc = w.clone(), [y.clone() for y in cache]
        for a, b in zip(to, of):
            if there[a]:
                for y in (ww, *wc):
                    y[p[a], 0, at[a]] = y[p[b], 0, at[b]]
        assert torch.equal(gw.cpu(), ww) and all(torch.equal(y.cpu(), z) for y, z in zip(c, wc))
    # recent rows on such a page
    u = t.clone()
    u[0, 4] = -5                                                           # keys 64 ... 79
    c, gw = cref.on_gpu(cache), w.cuda()
    A.attn_cache_evict(gw, c, u.cuda(), lens.cuda(), torch.tensor([20], dtype=torch.int32).cuda(), 16)
    j = torch.arange(4, 20)
    p, at = u[0, j // 16].long(), j % 16
    assert (c.k_scale.cpu()[p, 0, at] == 255).all() and (c.v_scale.cpu()[p, 0, at] == 255).all() and (gw.cpu()[p, 0, at] == 0).all()


def test_given_outputs_streams_and_graphs():
    import paper_2603_05451_amd as A
    cache, w, t, lens = _case(4, [500, 40, 777], 2, 128, 128, 4, 64)
    keep = torch.tensor([100, 50, 300], dtype=torch.int32)
    c, gw = cref.on_gpu(cache), w.cuda()
    gt, gl, gk = t.cuda(), lens.cuda(), keep.cuda()
    out = torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(A.attn_cache_evict_workspace_bytes(c, 3, t.shape[1]), dtype=torch.uint8, device="cuda")
    ww, wc = _want(w, cache, t, lens, keep, 20)

    def put():
        gw.copy_(w.cuda())
        out.zero_()
        for x, y in zip(c, cache):
            x.copy_(y.cuda())
        torch.cuda.synchronize()

    def right():
        return torch.equal(gw.cpu(), ww) and all(torch.equal(x.cpu(), y) for x, y in zip(c, wc)) and out.tolist() == [100, 40, 300]
    call = lambda **kw: A.attn_cache_evict(gw, c, gt, gl, gk, 20, lens_out=out, workspace=ws, **kw)
    assert call() is out and right()
    put()
    side = torch.cuda.Stream()
    call(stream=side)
    side.synchronize()
    assert right()
    graph = torch.cuda.CUDAGraph()
    put()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        put()
        graph.replay()
        torch.cuda.synchronize()
        assert right()
