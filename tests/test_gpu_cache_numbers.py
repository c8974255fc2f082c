"""GPU tests of attn_cache_fwd over values that are no finite numbers of the queries' type (a code and a scale beyond its range, e4m3's own
NaN, a page that is not there): they reach the queries that see their key, in their channel, and no other result by a bit."""
import pytest
import torch

from test_gpu_cache import _gen, _on_gpu, _random_cache, _table

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16

# (code, scale byte) of the least number that is infinite in the type, of the largest that is not, and of e4m3's NaN.
# 4 bits: 4 * 2^126 = 2^128, 6 * 2^125; 4 * 2^14 = 2^16, 6 * 2^13.  8 bits: 256 * 2^120, 448 * 2^119; 256 * 2^8, 448 * 2^7 (fp16's largest: 65504).
CODES = {("least", 4, BF): (6, 253), ("least", 8, BF): (0x78, 247), ("least", 4, HF): (6, 141), ("least", 8, HF): (0x78, 135),
         ("finite", 4, BF): (7, 252), ("finite", 8, BF): (0x7e, 246), ("finite", 4, HF): (7, 140), ("finite", 8, HF): (0x7e, 134),
         ("nan", 8, BF): (0x7f, 3), ("nan", 8, HF): (0x7f, 3)}

RUNS = {                                       # lens, Nq, H, Hkv, causal
    "short": ([70, 33, 4, 40, 64, 0], 4, 4, 2, True),
    "rows": ([70, 33, 5, 130], 5, 8, 2, True),                  # 20 rows of a group: two row blocks
    "all": ([70, 33, 129], 2, 4, 2, False),
    "divided": ([3001, 7, 1030], 3, 4, 2, True),
    "divided_rows": ([3001, 64, 1030], 9, 4, 2, True),
    "waves": ([300, 5] + [4, 37, 66] * 200, 4, 4, 2, True),     # more sequences than blocks
}


def _set(cache, i, at, ch, bits, code, scale):
    """The block of channel ch of a row: zeros and this code."""
    block = cache[i][at].view(-1, 32 * bits // 8)[ch // 32]
    block.zero_()
    if bits == 8:
        block[ch % 32] = code
    else:
        block[ch % 32 // 2] = code << 4 * (ch % 2)
    cache[i + 1][at][ch // 32] = scale


@pytest.mark.parametrize("run", list(RUNS))
@pytest.mark.parametrize("kind,bits,dtype", list(CODES))
@pytest.mark.parametrize("dqk,dv", [(64, 64), (96, 96), (128, 128), (192, 128), (256, 256)])
def test_reach_who_sees_them(run, kind, bits, dtype, dqk, dv):
    import paper_2603_05451_amd as A
    lens, Nq, H, Hkv, causal = RUNS[run]
    if run == "waves" and (dqk, dv) not in ((64, 64), (128, 128)):
        lens = lens[:302]                      # (as many blocks there)
    page, B = 16, len(lens)
    pages = sum(-(-n // page) for n in lens) + 2
    gen = _gen(dqk + bits)
    clean = _random_cache(gen, pages, page, Hkv, dqk, dv, bits)
    table = _table(gen, lens, page, pages)
    q = torch.randn(B, Nq, H, dqk, generator=gen).to(dtype)
    code, scale = CODES[kind, bits, dtype]
    minus = code | (8 if bits == 4 else 128)
    bad = [t.clone() for t in clean]
    odd = torch.zeros(B, Nq, H, dv, dtype=torch.bool)
    G = H // Hkv
    for b, n in enumerate(lens):
        for key, ch, x in ((n - 1, 5, code), (n - 1, 38, minus), (n - 3, dv - 1, code), (n - 2, 17, minus)):
            if key < 0:
                continue
            kvh, at = b % Hkv, (int(table[b, key // page]), b % Hkv, key % page)
            _set(bad, 2, at, ch, bits, x, scale)
            _set(clean, 2, at, ch, bits, 0, scale)
            for i in range(Nq):
                if not causal or key <= n - Nq + i:
                    odd[b, i, kvh * G:(kvh + 1) * G, ch] = True
    lens = torch.tensor(lens, dtype=torch.int32).cuda()
    go = lambda c: [t.cpu() for t in A.attn_cache_fwd(q.cuda(), _on_gpu(c), table.cuda(), lens, dqk ** -0.5, causal)]
    (o, lse), (want, want_lse) = go(bad), go(clean)
    assert torch.isfinite(want.float()).all() and torch.equal(lse, want_lse)
    if kind == "finite":
        # (fp16: below 2^16 2^8 n in the fp32 sums, 2^8 being the largest weight between two rescalings.  6 * 2^125 times such a weight may
        # pass 2^128 in them: the queries that see it may have an infinite result)
        assert dtype == BF or torch.isfinite(o.float()).all()
        odd &= o != want
    else:
        assert not torch.isfinite(o[odd].float()).any()
    assert torch.equal(torch.where(odd, 0, o), torch.where(odd, 0, want))


@pytest.mark.parametrize("bits", [4, 8])
def test_infinite_keys_behind_the_mask(bits):
    """A key that fp16 does not hold is hidden like any other."""
    import paper_2603_05451_amd as A
    gen = _gen(bits)
    clean = _random_cache(gen, 6, 16, 1, 128, 128, bits)
    table, lens = torch.randperm(6, generator=gen).int().view(1, 6), torch.tensor([90], dtype=torch.int32)
    bad = [t.clone() for t in clean]
    _set(bad, 0, (int(table[0, 89 // 16]), 0, 89 % 16), 40, bits, *CODES["least", bits, HF])
    q = torch.randn(1, 4, 2, 128, generator=gen).to(HF)
    (o, lse), (want, want_lse) = ([t.cpu() for t in A.attn_cache_fwd(q.cuda(), _on_gpu(c), table.cuda(), lens.cuda(), 0.1, True)] for c in (bad, clean))
    assert torch.equal(o[:, :3], want[:, :3]) and torch.equal(lse[..., :3], want_lse[..., :3])


@pytest.mark.parametrize("n", [49, 2049])
def test_page_outside_the_cache_behind_the_mask(n):
    """The last key's page is not there: the queries before it do without."""
    import paper_2603_05451_amd as A
    gen, pages = _gen(n), -(-n // 16)
    cache = _random_cache(gen, pages, 16, 2, 64, 64, 4)
    table, lens = torch.randperm(pages, generator=gen).int().view(1, pages), torch.tensor([n], dtype=torch.int32)
    q = torch.randn(1, 3, 4, 64, generator=gen).to(BF)
    bad = table.clone()
    bad[0, -1] = pages
    (o, lse), (want, want_lse) = ([t.cpu() for t in A.attn_cache_fwd(q.cuda(), _on_gpu(cache), t.cuda(), lens.cuda(), 0.1, True)] for t in (bad, table))
    assert torch.equal(o[:, :2], want[:, :2]) and torch.equal(lse[..., :2], want_lse[..., :2])
    assert torch.isnan(o[:, 2].float()).all() and torch.isnan(lse[..., 2]).all()
