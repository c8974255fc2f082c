"""The chunk, weight and eviction calls in a cache with more than 2^29 rows, whose weights pass 2^31 bytes: pages at its end against the same pages of a small
one, bit for bit; and eviction whose lists of places do not fit in LDS, of several sequences and heads."""
import pytest
import torch

import cache_reference as cref
from cache_reference import BF
from test_gpu_cache_evict import _case, _check

pytestmark = pytest.mark.gpu


def test_rows_behind_two_gigabytes_of_weights():
    import paper_2603_05451_amd as A
    Hkv, d, page, n, big = 1, 64, 16384, 40000, 33000
    assert big * Hkv * page * 4 > 2 ** 31
    g = cref.gen(1)
    small = A.AttnCache(*(x.cuda() for x in cref.random_cache(g, 3, page, Hkv, d, d, 4)))
    large = A.AttnCache(*(torch.empty(big, Hkv, page, x.shape[3], dtype=torch.uint8, device="cuda") for x in small))
    w, wl = torch.rand(3, Hkv, page, generator=g).cuda(), torch.empty(big, Hkv, page, device="cuda")
    at = torch.tensor([big - 1, big - 3, big - 2])
    for x, y in (*zip(small, large), (w, wl)):
        y[at.cuda()] = x
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q = torch.randn(40, 4, d, generator=g).to(BF).cuda()
    results = []
    for c, weights, table in ((small, w, torch.arange(3)), (large, wl, at)):
        table = table.int().view(1, 3).cuda()
        o, lse = A.attn_cache_chunk_fwd(q, c, table, i(0, 40), i(n), 0.125, True)
        A.attn_cache_weigh(q, lse, weights, c, table, i(n), 0.125, True, cu_seqlens=i(0, 40), fresh=True)
        few, l3 = A.attn_cache_fwd(q[None, :3], c, table, i(n), 0.125, True)
        A.attn_cache_weigh(q[None, :3], l3, weights, c, table, i(n), 0.125, True)
        left = A.attn_cache_evict(weights, c, table, i(n), i(12000), 100)
        results.append((o, lse, few, l3, left, *(x[table[0].long()] for x in (*c, weights))))
    del large, wl, c, weights
    torch.cuda.empty_cache()                                   # 39 GB
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_evict_lists_in_the_workspace_and_in_lds():
    """Tables of more than 32 768 rows: sequences that need the workspace for their lists next to such that do not."""
    cache, w, t, lens = _case(3, [33000, 500, 40001, 0, 32800], 2, 64, 64, 4, 256)
    _check(cache, w, t, lens, [20000, 100, 39000, 5, 32700], 40)
