"""The chunk, weight and eviction calls in a cache whose codes pass 4 GiB and whose rows pass 2^31 bytes of weights: pages at its end against the same
pages of a small one, bit for bit."""
import pytest
import torch

import cache_reference as cref
from cache_reference import BF

pytestmark = pytest.mark.gpu


def test_pages_behind_four_gigabytes():
    import paper_2603_05451_amd as A
    Hkv, d, page, n = 2, 256, 1024, 3000
    big = 8800                                                 # pages: 18 M rows, 4.6 GB of codes each way
    assert big * Hkv * page * d > 2 ** 32 + 2 ** 28
    g = cref.gen(1)
    small = A.AttnCache(*(x.cuda() for x in cref.random_cache(g, 4, page, Hkv, d, d, 8)))
    large = A.AttnCache(*(torch.empty(big, Hkv, page, x.shape[3], dtype=torch.uint8, device="cuda") for x in small))
    w, wl = torch.rand(4, Hkv, page, generator=g).cuda(), torch.empty(big, Hkv, page, device="cuda")
    at = torch.tensor([big - 1, 0, big - 3, big - 2])
    for x, y in ((*zip(small, large), (w, wl))):
        y[at.cuda()] = x
    q, cu = torch.randn(40, 4, d, generator=g).to(BF).cuda(), torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    lens, keep = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([1200], dtype=torch.int32, device="cuda")
    results = []
    for c, weights, table in ((small, w, torch.arange(4)), (large, wl, at)):
        table = table.int().view(1, 4).cuda()
        o, lse = A.attn_cache_chunk_fwd(q, c, table, cu, lens, 0.06, True)
        A.attn_cache_weigh(q, lse, weights, c, table, lens, 0.06, True, cu_seqlens=cu, fresh=True)
        _, few = A.attn_cache_chunk_fwd(q[:3], c, table, torch.tensor([0, 3], dtype=torch.int32, device="cuda"), lens, 0.06, True)
        A.attn_cache_weigh(q[:3], few, weights, c, table, lens, 0.06, True, cu_seqlens=torch.tensor([0, 3], dtype=torch.int32, device="cuda"))
        left = A.attn_cache_evict(weights, c, table, lens, keep, 100)
        results.append((o, lse, few, left, *(x[table[0].long()] for x in (*c, weights))))
    assert all(torch.equal(x, y) for x, y in zip(*results))
