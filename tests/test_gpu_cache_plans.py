"""GPU tests of how the chunk and weight calls share out batches with more sequences than a wave has lanes, more work than blocks, and tables wider than any
sequence: results against 64 bits (tolerances: cache_reference.py)."""
import pytest
import torch

import cache_reference as cref
from cache_reference import BF, HF
from test_gpu_cache_chunk import _case, _run
from test_gpu_cache_weigh import _check, _weights

pytestmark = pytest.mark.gpu


def _widen(t, width):
    """The same pages in a wider table, with nonsense behind them."""
    wide = torch.randint(-2 ** 31, 2 ** 31 - 1, (t.shape[0], width), generator=cref.gen(1)).int()
    wide[:, :t.shape[1]] = t
    return wide


def _both(q, cache, t, cu, lens, scale, causal, bits, sequences=None):
    """Attention, then the weights of its keys (with its own lse); both checked."""
    import paper_2603_05451_amd as A
    c = cref.on_gpu(cache)
    o, lse = _run(q, c, t, cu, lens, scale, causal)
    cref.check_attention(q, cache, t, cu, lens, scale, causal, o.cpu(), lse.cpu(), bits, sequences)
    w = _weights(cref.gen(4), cache)
    got = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse, got, c, t.cuda(), lens.cuda(), scale, causal, cu_seqlens=cu.cuda(), fresh=causal)
    _check(q, lse.cpu(), w, got.cpu(), cache, t, cu, lens, scale, causal, causal, bits)


# more than 64 sequences: single tokens, some without queries or keys, and from 65 on such whose rows and keys are divided
_SHORT = [(1, 40), (1, 129), (0, 30), (3, 70), (1, 0), (2, 1)] * 12
MANY = _SHORT[:70] + [(300, 520), (1, 900), (40, 1700)] + _SHORT[:60] + [(9, 2500), (150, 150), (64, 1100), (33, 3)] + _SHORT[:5]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dqk,dv,Hkv,G,bits,dtype", [(64, 64, 2, 2, 8, HF), (128, 128, 1, 4, 4, BF), (256, 256, 1, 2, 4, BF)])
def test_more_sequences_than_lanes(dqk, dv, Hkv, G, bits, dtype, causal):
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(dqk, MANY, Hkv, G, dqk, dv, bits, 32, dtype)
    c = cref.on_gpu(cache)
    B, T, H = len(MANY), q.shape[0], Hkv * G
    assert A.attn_cache_chunk_workspace_bytes(c, B, T, H, t.shape[1]) > 256 and A.attn_cache_weigh_workspace_bytes(c, B, T, H, t.shape[1], True) > 256
    _both(q, cache, t, cu, lens, dqk ** -0.5, causal, bits)


@pytest.mark.parametrize("width", [200, 3000])
def test_table_wider_than_any_sequence(width):
    """Shares, parts and workspaces go by the table's width: the results do not."""
    seqs = [(1, 40), (70, 300), (0, 90), (5, 31), (130, 1000), (1, 800)]
    q, cache, t, cu, lens = _case(3, seqs, 2, 4, 128, 128, 4, 16, BF)
    _both(q, cache, _widen(t, width), cu, lens, 0.09, True, 4)


@pytest.mark.parametrize("dqk,dv,bits,dtype", [(64, 64, 4, HF), (128, 128, 8, BF), (192, 128, 4, BF)])
def test_many_rows_divided(dqk, dv, bits, dtype):
    """Sequences of more than 128 rows whose keys are divided."""
    q, cache, t, cu, lens = _case(dqk, [(50, 9001), (33, 2500), (1, 700)], 2, 4, dqk, dv, bits, 64, dtype)
    _both(q, cache, t, cu, lens, dqk ** -0.5, True, bits)


def test_lengths_beyond_a_table_of_many_sequences():
    """Sequences that fill their row of the table, with a length far beyond it, among more than 64."""
    seqs = [(4, 50)] * 66 + [(5, 128)] + [(1, 90)] * 8 + [(70, 128)]
    q, cache, t, cu, lens = _case(5, seqs, 2, 2, 64, 64, 4, 16, BF)
    assert t.shape[1] * 16 == 128
    lens[66], lens[75] = 2 ** 31 - 1, 129
    _both(q, cache, t, cu, lens, 0.125, True, 4)


@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_more_work_than_blocks(causal):
    """More than 1024 units, so that blocks take several: of few rows and of many in turn, some of these in shares."""
    Hkv, G, d = 8, 4, 64
    seqs = [(9 + i % 7, 4000 - 37 * i) if i % 3 else (1 + i % 8, 1500 + 100 * i) for i in range(30)] + [(500, 900), (0, 50), (8, 4000), (20, 257)]
    few = [nq * G <= 32 for nq, _ in seqs]
    many = [(-(-n // 256), -(-nq * G // 128)) for (nq, n), f in zip(seqs, few) if not f and nq]
    share = max(2, -(-sum(a * b for a, b in many) * Hkv // 512))
    assert sum(a * max(1, (b + share // 2) // share) for a, b in many) * Hkv > 1024 and any(b >= 2 * share for _, b in many) and any(few)
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(11, seqs, Hkv, G, d, d, 4, 64, BF)
    c = cref.on_gpu(cache)
    _, lse = _run(q, c, t, cu, lens, 0.125, causal)
    w = _weights(cref.gen(4), cache)
    got = w.cuda()
    A.attn_cache_weigh(q.cuda(), lse, got, c, t.cuda(), lens.cuda(), 0.125, causal, cu_seqlens=cu.cuda(), fresh=causal)
    _check(q, lse.cpu(), w, got.cpu(), cache, t, cu, lens, 0.125, causal, causal, 4)
