"""The chunk, weight and eviction calls in the run that they are made for: prompts served in chunks beside tokens, the cache kept within a budget; as a
captured graph; and the native marshalling of the three against the Python text."""
import pytest
import torch

import cache_reference as cref
import ops_reference as ref
from cache_reference import BF, HF
from test_gpu_binding import _both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,dtype", [(4, BF), (8, HF)])
def test_serving_within_a_budget(bits, dtype):
    """Three requests (one joins late): chunks of their prompts and single tokens in mixed batches, a step of attn_cache_fwd among them; after every step what
    its keys weighed, and eviction down to a budget.  Every result against 64 bits on what the cache holds by definition; which rows leave,
    exactly, by the weights as the GPU has them."""
    import paper_2603_05451_amd as A
    H, Hkv, d, page, scale, budget, recent, B = 8, 2, 64, 16, 64 ** -0.5, 48, 6, 3
    g = cref.gen(bits)
    cache = A.attn_cache_new(30, page, Hkv, d, d, bits)
    weights = A.attn_cache_weights(cache)
    weights.fill_(1e9)                                         # what a former owner of the pages left: `fresh` sets the new rows' weights
    table = torch.randperm(30, generator=g).int().view(B, 10)
    held = [[torch.empty(0, Hkv, d, dtype=torch.float64) for _ in range(2)] for _ in range(B)]
    want = [torch.empty(0, Hkv, dtype=torch.float64) for _ in range(B)]
    off = [torch.empty(0, Hkv, dtype=torch.float64) for _ in range(B)]
    slot = lambda b, j: int(table[b, j // page]) * page + j % page
    at = lambda b, n: (table[b, torch.arange(n) // page].long(), torch.arange(n) % page)

    for step, news in enumerate([[70, 40, 0], [1, 33, 50], [1, 1, 1], [4, 4, 4], [30, 0, 65], [1, 1, 1]]):
        T = sum(news)
        q, k, v = (torch.randn(T, h, d, generator=g).to(dtype) for h in (H, Hkv, Hkv))
        cu = torch.tensor([0, *torch.tensor(news).cumsum(0)], dtype=torch.int32)
        before = [x[0].shape[0] for x in held]
        slots = torch.tensor([slot(b, before[b] + i) for b in range(B) for i in range(news[b])], dtype=torch.int32)
        A.attn_cache_write(k.cuda(), v.cuda(), slots.cuda(), cache)
        lens = torch.tensor([n + m for n, m in zip(before, news)], dtype=torch.int32)
        equal = len(set(news)) == 1 and step > 2               # a decode or draft step: the call for few queries
        if equal:
            Nq = news[0]
            o, lse = A.attn_cache_fwd(q.cuda().view(B, Nq, H, d), cache, table.cuda(), lens.cuda(), scale, True)
            A.attn_cache_weigh(q.cuda().view(B, Nq, H, d), lse, weights, cache, table.cuda(), lens.cuda(), scale, True, fresh=True)
            o, lse = o.view(T, H, d).cpu(), lse.transpose(0, 1).reshape(H, T).cpu()
        else:
            o, lse = A.attn_cache_chunk_fwd(q.cuda(), cache, table.cuda(), cu.cuda(), lens.cuda(), scale, True)
            A.attn_cache_weigh(q.cuda(), lse, weights, cache, table.cuda(), lens.cuda(), scale, True, cu_seqlens=cu.cuda(), fresh=True)
            o, lse = o.cpu(), lse.cpu()
        now = [x.cpu() for x in cache]
        cref.check_attention(q, now, table, cu, lens, scale, True, o, lse, bits)
        for b in range(B):
            i0, i1, n = int(cu[b]), int(cu[b + 1]), int(lens[b])
            for i, x in enumerate((k, v)):
                held[b][i] = torch.cat((held[b][i], ref.values(*ref.quantise(x[i0:i1], bits), bits)))
                assert torch.equal(held[b][i], cref.rows(now, table, b, n, bits)[i])
            if news[b]:
                got, e = cref.weigh(q[i0:i1].double(), lse[:, i0:i1], held[b][0], scale, True)
                pad = lambda x: torch.cat((x, torch.zeros(news[b], Hkv, dtype=torch.float64)))
                want[b], off[b] = pad(want[b]) + got, pad(off[b]) + e
            p, a = at(b, n)
            mine = weights.cpu()[p, :, a].double()
            assert ((mine - want[b]).abs() <= off[b] + (step + 1) * cref.STEP * want[b]).all()
            want[b] = mine                                     # the sums as they are, exactly, from here on
            off[b] = torch.zeros_like(mine)
        had = weights.cpu()
        left = A.attn_cache_evict(weights, cache, table.cuda(), lens.cuda(), torch.full((B,), budget, dtype=torch.int32, device="cuda"), recent)
        assert left.tolist() == [min(int(n), budget) for n in lens]
        for b in range(B):
            n = int(lens[b])
            p, a = at(b, n)
            for h in range(Hkv):
                to, of = cref.places(had[p, h, a].tolist(), n, budget, recent)
                for x in (*held[b], want[b]):
                    x[to, h] = x[of, h].clone()
            keep = min(n, budget)
            held[b], want[b], off[b] = [x[:keep] for x in held[b]], want[b][:keep], off[b][:keep]
            p, a = at(b, keep)
            assert torch.equal(weights.cpu()[p, :, a].double(), want[b])
            got = cref.rows([x.cpu() for x in cache], table, b, keep, bits)
            assert torch.equal(got[0], held[b][0]) and torch.equal(got[1], held[b][1])


def test_a_step_in_a_graph():
    """Attention, weights and eviction of a chunk, captured once and replayed on other requests, with eager work between: the eager calls' bits."""
    import paper_2603_05451_amd as A
    g = cref.gen(9)
    B, T, H, Hkv, d, page, width = 4, 90, 8, 2, 128, 16, 40
    cache = A.AttnCache(*(x.cuda() for x in cref.random_cache(g, B * width, page, Hkv, d, d, 4)))
    weights = A.attn_cache_weights(cache)
    s = {"q": torch.zeros(T, H, d, dtype=BF, device="cuda"), "cu": torch.zeros(B + 1, dtype=torch.int32, device="cuda"), "lens": torch.zeros(B, dtype=torch.int32, device="cuda"),
         "table": torch.zeros(B, width, dtype=torch.int32, device="cuda"), "keep": torch.zeros(B, dtype=torch.int32, device="cuda"),
         "o": torch.zeros(T, H, d, dtype=BF, device="cuda"), "lse": torch.zeros(H, T, device="cuda"), "left": torch.zeros(B, dtype=torch.int32, device="cuda")}
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in
          (A.attn_cache_chunk_workspace_bytes(cache, B, T, H, width), A.attn_cache_weigh_workspace_bytes(cache, B, T, H, width, True), A.attn_cache_evict_workspace_bytes(cache, B, width))]

    def step():
        A.attn_cache_chunk_fwd(s["q"], cache, s["table"], s["cu"], s["lens"], 0.09, True, o=s["o"], lse=s["lse"], workspace=ws[0])
        A.attn_cache_weigh(s["q"], s["lse"], weights, cache, s["table"], s["lens"], 0.09, True, cu_seqlens=s["cu"], fresh=True, workspace=ws[1])
        A.attn_cache_evict(weights, cache, s["table"], s["lens"], s["keep"], 4, lens_out=s["left"], workspace=ws[2])

    fresh = [x.clone() for x in cache]
    requests = []
    for news, keys in (([40, 1, 0, 7], [600, 300, 50, 7]), ([1, 1, 1, 80], [500, 20, 333, 80]), ([0, 64, 20, 6], [10, 640, 90, 6])):
        requests.append((torch.randn(T, H, d, generator=g).to(BF), torch.tensor([0, *torch.tensor(news).cumsum(0)]).int(), torch.tensor(keys).int(),
                         torch.randperm(B * width, generator=g).int().view(B, width), torch.tensor([keys[0] // 2, 15, 1000, 5]).int()))

    def put(r):
        for name, x in zip(("q", "cu", "lens", "table", "keep"), r):
            s[name].copy_(x.cuda())
        for x, y in zip(cache, fresh):
            x.copy_(y)
        weights.zero_()
        s["o"].zero_()
        s["lse"].zero_()

    def state():
        return [x.clone() for x in (*cache, weights, s["o"], s["lse"], s["left"])]
    want = []
    for r in requests:
        put(r)
        step()
        want.append(state())
    put(requests[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 0, 2, 2, 0, 1):
        put(requests[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(state(), want[i]))


def _inputs(A, dtype=BF):
    c = A.AttnCache(*(x.cuda() for x in cref.random_cache(cref.gen(1), 8, 16, 2, 64, 64, 4)))
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q = torch.randn(18, 4, 64, generator=cref.gen(2)).to(dtype).cuda()
    return q, c, torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3), i(0, 9, 18), i(40, 17), i(20, 10)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_same_outputs_by_both_bindings(monkeypatch, dtype):
    def calls(A):
        q, c, table, cu, lens, keep = _inputs(A, dtype)
        o, lse = A.attn_cache_chunk_fwd(q, c, table, cu, lens, 0.125, True)
        wide = torch.zeros(18, 6, 72, dtype=dtype, device="cuda")
        wide[:, 1:5, :64] = q
        mine = torch.zeros(4, 18, 64, dtype=dtype, device="cuda").transpose(0, 1)
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        r = A.attn_cache_chunk_fwd(wide[:, 1:5, :64], c, table, cu, lens, 0.125, False, o=mine, lse=torch.zeros_like(lse), workspace=ws)
        assert r[0] is mine
        w = A.attn_cache_weights(c)
        assert A.attn_cache_weigh(q, lse, w, c, table, lens, 0.125, True, cu_seqlens=cu, fresh=True) is w
        few = w.clone()
        q4 = q.view(2, 9, 4, 64)[:, :2]
        _, l4 = A.attn_cache_fwd(q4, c, table, lens, 0.125, True)
        A.attn_cache_weigh(q4, l4, few, c, table, lens, 0.125, True, workspace=ws)
        left = A.attn_cache_evict(w, c, table, lens, keep, 3)
        out = torch.zeros(2, dtype=torch.int32, device="cuda")
        assert A.attn_cache_evict(few, c, table, lens, keep, 0, lens_out=out, workspace=ws) is out
        return [o, lse, *r, w, few, left, out, *c]

    native, python, results = _both(monkeypatch, calls)
    assert [n for n, r in results] == ["cache_chunk_fwd"] * 2 + ["cache_weigh", "cache_fwd", "cache_weigh", "cache_evict", "cache_evict"]
    assert all(r is not None for n, r in results)
    for i, (x, y) in enumerate(zip(native, python)):
        assert x.shape == y.shape and x.stride() == y.stride() and x.dtype == y.dtype and torch.equal(x, y), i


def test_same_refusals_by_both_bindings(monkeypatch):
    import paper_2603_05451_amd as A
    q, c, table, cu, lens, keep = _inputs(A)
    lse, w = torch.zeros(4, 18, device="cuda"), A.attn_cache_weights(c)
    q4, l4 = q.view(2, 9, 4, 64), torch.zeros(2, 4, 9, device="cuda")
    chunk = lambda q_=q, c_=c, t=table, u=cu, n=lens, s=0.1, **k: lambda A: A.attn_cache_chunk_fwd(q_, c_, t, u, n, s, True, **k)
    weigh = lambda q_=q, l=lse, w_=w, c_=c, t=table, n=lens, s=0.1, u=cu, **k: lambda A: A.attn_cache_weigh(q_, l, w_, c_, t, n, s, True, cu_seqlens=u, **k)
    evict = lambda w_=w, c_=c, t=table, n=lens, k=keep, r=3, **x: lambda A: A.attn_cache_evict(w_, c_, t, n, k, r, **x)
    byte = torch.empty(300, dtype=torch.uint8, device="cuda")
    for i, call in enumerate([chunk(q4), chunk(q[:, :3]), chunk(q.float()), chunk(q[..., :32]), chunk(t=table[:1]), chunk(t=table.long()), chunk(u=cu[:2]), chunk(u=cu.cpu()),
                              chunk(n=lens[:1]), chunk(s=-1.0), chunk(o=q[:9]), chunk(lse=l4), chunk(workspace=lens), chunk(workspace=byte[1:257]),
                              chunk(c_=c._replace(k=c.v_scale)), weigh(q4), weigh(u=None), weigh(q4, l4[:1], u=None), weigh(q4[:1], l4, u=None), weigh(l=l4), weigh(w_=w[:4]),
                              weigh(w_=w.double()), weigh(w_=w.cpu()), weigh(s=0.0), weigh(u=cu[:1]), weigh(n=keep.cpu()), weigh(workspace=w), evict(w[1:]), evict(t=table[:1]),
                              evict(n=lens[:1]), evict(k=keep[:1]), evict(k=keep.long()), evict(r=-1), evict(lens_out=lens), evict(lens_out=keep), evict(lens_out=lens[:1]),
                              evict(workspace=byte[:256])]):
        def said(A):
            with pytest.raises((ValueError, A.AttnError)) as e:
                call(A)
            return type(e.value), str(e.value)
        native, python, results = _both(monkeypatch, said)
        assert native == python, i
        assert all(r is None or (type(r) is int and r < 0 and native[0].__name__ == "AttnError") for n, r in results), i


def test_foreign_streams_and_devices():
    """Tensors of another device than the current one are refused; a stream of the caller's gives the plain call's results."""
    import paper_2603_05451_amd as A
    q, c, table, cu, lens, keep = _inputs(A)
    o, lse = A.attn_cache_chunk_fwd(q, c, table, cu, lens, 0.125, True)
    w = A.attn_cache_weigh(q, lse, A.attn_cache_weights(c), c, table, lens, 0.125, True, cu_seqlens=cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = A.attn_cache_chunk_fwd(q, c, table, cu, lens, 0.125, True, stream=side)
    with torch.cuda.stream(side):
        w2 = A.attn_cache_weights(c)
    A.attn_cache_weigh(q, r[1], w2, c, table, lens, 0.125, True, cu_seqlens=cu, stream=side)
    mine = A.AttnCache(*(x.clone() for x in c))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(r[0], o) and torch.equal(r[1], lse) and torch.equal(w, w2)
    side.wait_stream(torch.cuda.current_stream())
    left = A.attn_cache_evict(w2, mine, table, lens, keep, 3, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(left, A.attn_cache_evict(w, c, table, lens, keep, 3)) and all(torch.equal(x, y) for x, y in zip(mine, c)) and torch.equal(w, w2)
    for f in (lambda: A.attn_cache_chunk_fwd(q, c, table.cpu(), cu, lens, 0.125, True), lambda: A.attn_cache_evict(w.cpu(), c, table, lens, keep, 3)):
        with pytest.raises(ValueError):
            f()
