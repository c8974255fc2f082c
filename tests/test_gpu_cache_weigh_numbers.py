"""GPU tests of attn_cache_weigh with queries that are left out and with numbers that are not finite (tolerances: cache_reference.weigh)."""
import math

import pytest
import torch

import cache_reference as cref
from cache_reference import BF, HF
from test_gpu_cache_chunk import MIX, _case
from test_gpu_cache_weigh import _check, _lse, _weights

pytestmark = pytest.mark.gpu


def _leave_out(q, lse, rows):
    """Rows of q that are no numbers any more (each in its way), whose lse says that they are to add nothing."""
    for i, t in enumerate(rows):
        q[t] = (math.nan, math.inf, -math.inf)[i % 3]
        lse[:, t] = -math.inf


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dqk,dv,bits", [(64, 64, 8), (96, 96, 4), (128, 128, 4), (192, 128, 8), (256, 256, 4)])
def test_queries_left_out(dqk, dv, bits, causal):
    """A query with lse = -inf adds nothing, whatever its row of q holds: some of a sequence's, all of one's, the last one."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(dqk, [*MIX, (150, 400), (40, 90)], 2, 3, dqk, dv, bits, 16, BF)
    scale = dqk ** -0.5
    lse = _lse(q, cache, t, cu, lens, scale, causal, bits)
    out = torch.randperm(q.shape[0], generator=cref.gen(3))[:q.shape[0] // 4].tolist()
    out += [*range(int(cu[-3]) + 64, int(cu[-3]) + 100), q.shape[0] - 1, *range(int(cu[4]), int(cu[5])), int(cu[5])]
    _leave_out(q, lse, out)
    w = _weights(cref.gen(1), cache)
    got = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse.cuda(), got, cref.on_gpu(cache), t.cuda(), lens.cuda(), scale, causal, cu_seqlens=cu.cuda(), fresh=True)
    _check(q, lse, w, got.cpu(), cache, t, cu, lens, scale, causal, True, bits)


@pytest.mark.parametrize("Nq", [3, 40])
def test_queries_left_out_of_an_equal_batch(Nq):
    """A batch of drafts of different lengths, padded in front."""
    import paper_2603_05451_amd as A
    B, Hkv, G = 4, 2, 4
    H = Hkv * G
    q, cache, t, cu, lens = _case(7, [(Nq, n) for n in (900, 64, 70, 333)], Hkv, G, 128, 128, 4, 64, HF)
    lse = _lse(q, cache, t, cu, lens, 0.09, True, 4)
    _leave_out(q, lse, [b * Nq + i for b in range(B) for i in range(min(b, Nq))])
    w = _weights(cref.gen(2), cache)
    got = w.cuda()
    A.attn_cache_weigh(q.cuda().view(B, Nq, H, 128), lse.view(H, B, Nq).transpose(0, 1).contiguous().cuda(), got, cref.on_gpu(cache), t.cuda(), lens.cuda(), 0.09, True)
    _check(q, lse, w, got.cpu(), cache, t, cu, lens, 0.09, True, False, 4)


@pytest.mark.parametrize("nq", [3, 90])
def test_a_nan_key_through_the_calls(nq):
    """With the attention call's own lse: the queries that see a NaN key have lse = NaN, and every key that they see has the weight NaN; the other KV head's
    keys and the other sequence's are as without it.  Eviction takes the NaNs for the greatest, the first of them first."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(8, [(nq, 120), (nq, 100)], 2, 2, 64, 64, 4, 16, BF)
    p, at = int(t[0, 100 // 16]), 100 % 16
    cache[1][p, 1, at] = 255
    c = cref.on_gpu(cache)
    _, lse = A.attn_cache_chunk_fwd(q.cuda(), c, t.cuda(), cu.cuda(), lens.cuda(), 0.125, True)
    first = max(0, 100 - (120 - nq))                           # of the queries that see it
    nan = torch.isnan(lse.cpu())
    assert nan[2:, first:nq].all() and int(nan.sum()) == 2 * (nq - first)
    got = A.attn_cache_weigh(q.cuda(), lse, A.attn_cache_weights(c), c, t.cuda(), lens.cuda(), 0.125, True, cu_seqlens=cu.cuda(), fresh=True)
    slots = lambda b, n: (t[b, torch.arange(n) // 16].long(), torch.arange(n) % 16)
    mine = [got.cpu()[i, :, j] for i, j in (slots(0, 120), slots(1, 100))]
    assert torch.isnan(mine[0][:, 1]).all() and torch.isfinite(mine[0][:, 0]).all() and torch.isfinite(mine[1]).all()
    for b, n, heads in ((0, 120, slice(0, 1)), (1, 100, slice(0, 2))):
        k, _ = cref.rows(cache, t, b, n, 4)
        rows = slice(int(cu[b]), int(cu[b + 1]))
        h = slice(0, 2 * len(range(2)[heads]))
        want, off = cref.weigh(q[rows, h].double(), lse.cpu()[h, rows], k[:, heads], 0.125, True)
        assert ((mine[b][:, heads].double() - want).abs() <= off + cref.STEP * want).all()
    keep = torch.tensor([50, 100], dtype=torch.int32).cuda()
    before = got.cpu()
    A.attn_cache_evict(got, c, t.cuda(), lens.cuda(), keep, 5)
    i, j = slots(0, 50)
    assert torch.isnan(got.cpu()[i, 1, j]).all() and torch.equal(c.k.cpu()[i[:45], 1, j[:45]], cache[0][i[:45], 1, j[:45]])
    left = before[slots(0, 120)[0], 0, slots(0, 120)[1]]
    to, of = cref.places(left.tolist(), 120, 50, 5)
    left[to] = left[of].clone()
    assert torch.equal(got.cpu()[i, 0, j], left[:50])


@pytest.mark.parametrize("nq", [2, 70])
def test_an_infinite_key(nq):
    """A key beyond fp16's range whose scores are all -inf weighs nothing; with a score of +inf it is NaN."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(13, [(nq, 100)], 1, 2, 64, 64, 8, 16, HF)
    q = -q.abs() - 1
    p, at = int(t[0, 20 // 16]), 20 % 16
    cache[0][p, 0, at], cache[1][p, 0, at] = 0x70, 127 + 9     # 128 * 2^9 = 2^16 everywhere
    for sign in (1, -1):
        c = cref.on_gpu(cache)
        lse = A.attn_cache_chunk_fwd((sign * q).cuda(), c, t.cuda(), cu.cuda(), lens.cuda(), 0.125, True)[1]
        w = A.attn_cache_weigh((sign * q).cuda(), lse, A.attn_cache_weights(c), c, t.cuda(), lens.cuda(), 0.125, True, cu_seqlens=cu.cuda(), fresh=True).cpu()
        if sign == 1:
            assert torch.isfinite(lse).all() and w[p, 0, at] == 0 and torch.isfinite(w).all()
        else:
            assert not torch.isfinite(lse).any() and torch.isnan(w[p, 0, at])
