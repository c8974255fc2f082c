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
