"""GPU tests of attn_cache_fwd where a sequence's keys are divided among blocks and merged: every head dim and both code widths against
64 bits (the tolerance is that of test_gpu_cache.py), one query and several, one and two row blocks; a long sequence, whose rows' parts
a block of the merge deals to all its threads, and mixed lengths, of which it takes several rows."""
import pytest
import torch

from test_gpu_cache import DIMS, _gen, _on_gpu, _random_cache, _run, _table

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("Nq,H,Hkv,dtype", [(1, 4, 1, BF), (3, 6, 2, HF), (5, 8, 2, BF)])
@pytest.mark.parametrize("lens", [[5003], [1500, 3, 0, 257, 1025, 1999]])
def test_against_64_bits(lens, Nq, H, Hkv, dtype, dqk, dv, bits):
    _run(Nq + bits, lens, Nq, H, Hkv, dqk, dv, bits, 32, dtype, True, view=Nq == 3)


@pytest.mark.parametrize("bits,dqk,dv", [(4, 128, 128), (8, 96, 96)])
@pytest.mark.parametrize("Nq,H,Hkv", [(1, 2, 1), (5, 8, 2)])
def test_nan_blocks_in_the_chunks(Nq, H, Hkv, dqk, dv, bits):
    """A value block that is NaN in the first, a middle and the last chunk: 32 channels of the heads and queries that see it."""
    import paper_2603_05451_amd as A
    gen, lens = _gen(Nq + dqk), [1500, 1999, 40]
    cache = _random_cache(gen, 130, 32, Hkv, dqk, dv, bits)
    table = _table(gen, lens, 32, 130)
    q, n = torch.randn(3, Nq, H, dqk, generator=gen).to(BF), torch.tensor(lens, dtype=torch.int32).cuda()
    go = lambda c: [t.cpu() for t in A.attn_cache_fwd(q.cuda(), _on_gpu(c), table.cuda(), n, 0.1, True)]
    want, want_lse = go(cache)
    for b, key, block in ((0, 10, 0), (1, 700, 2), (1, 1999 - 1, 1), (0, 1500 - 3, 1)):
        bad = [t.clone() for t in cache]
        kvh = b % Hkv
        bad[3][int(table[b, key // 32]), kvh, key % 32, block] = 255
        o, lse = go(bad)
        odd = torch.zeros(o.shape, dtype=torch.bool)
        first = max(0, key - (lens[b] - Nq))                     # the first query that sees the key
        odd[b, first:, kvh * (H // Hkv):(kvh + 1) * (H // Hkv), 32 * block:32 * block + 32] = True
        assert torch.equal(lse, want_lse) and torch.isnan(o[odd].float()).all()
        assert torch.equal(torch.where(odd, 0, o), torch.where(odd, 0, want))


def test_rows_and_repeats():
    """More rows than a group's two blocks, divided: against 64 bits, and the same bits again."""
    import paper_2603_05451_amd as A
    _run(11, [2500, 300, 0], 7, 16, 2, 128, 128, 4, 64, BF, True)
    gen, lens = _gen(12), [2100, 900, 5]
    cache = _on_gpu(_random_cache(gen, 60, 64, 2, 64, 64, 4))
    table = _table(gen, lens, 64, 60).cuda()
    q, n = torch.randn(3, 2, 8, 64, generator=gen).to(HF).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    assert A.attn_cache_workspace_bytes(cache, 3, 2, 8, table.shape[1]) > 256        # (divided)
    first = [t.clone() for t in A.attn_cache_fwd(q, cache, table, n, 0.1, True)]
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(A.attn_cache_fwd(q, cache, table, n, 0.1, True), first))
