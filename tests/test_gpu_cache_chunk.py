"""GPU tests of attn_cache_chunk_fwd against the definition in 64 bits on what the cache holds (tolerances: cache_reference.py)."""
import itertools
import math

import pytest
import torch

import cache_reference as cref
import ops_reference as ref
from cache_reference import BF, DIMS, HF

pytestmark = pytest.mark.gpu

# (queries, keys): single tokens, fewer keys than queries, whole prompts, sequences without queries or keys, tiles of 32, 64 and 128 and one more or less
MIX = [(1, 1), (5, 3), (33, 33), (0, 20), (64, 200), (1, 300), (130, 131), (7, 0), (31, 64), (32, 65), (128, 128), (2, 2)]


def _case(seed, seqs, Hkv, G, dqk, dv, bits, page, dtype, pad=0, spare=2):
    g = cref.gen(seed)
    lens = [n for _, n in seqs]
    cu = torch.tensor([0, *itertools.accumulate(nq for nq, _ in seqs)], dtype=torch.int32)
    pages = sum(-(-max(n, 0) // page) for n in lens) + spare
    cache = cref.random_cache(g, pages, page, Hkv, dqk, dv, bits)
    t = cref.table(g, lens, page, pages)
    q = torch.randn(int(cu[-1]) + pad, Hkv * G, dqk, generator=g).to(dtype)
    return q, cache, t, cu, torch.tensor(lens, dtype=torch.int32)


def _run(q, cache, t, cu, lens, scale, causal, **kw):
    import paper_2603_05451_amd as A
    c = cache if isinstance(cache, A.AttnCache) else cref.on_gpu(cache)
    return A.attn_cache_chunk_fwd(q.cuda(), c, t.cuda(), cu.cuda(), lens.cuda(), scale, causal, **kw)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dqk,dv", DIMS)
def test_mixed_batch(dqk, dv, dtype, bits, causal):
    q, cache, t, cu, lens = _case(dqk + bits, MIX, 2, 3, dqk, dv, bits, 16, dtype)
    o, lse = _run(q, cache, t, cu, lens, dqk ** -0.5, causal)
    assert o.shape == (q.shape[0], 6, dv) and lse.shape == (6, q.shape[0]) and o.dtype == dtype
    cref.check_attention(q, cache, t, cu, lens, dqk ** -0.5, causal, o.cpu(), lse.cpu(), bits)


@pytest.mark.parametrize("Hkv,G,page", [(1, 1, 64), (1, 8, 256), (8, 4, 32), (5, 7, 128)])
def test_heads_and_pages(Hkv, G, page):
    q, cache, t, cu, lens = _case(Hkv * G, [(40, 700), (3, 1000), (129, 129)], Hkv, G, 128, 128, 4, page, BF)
    o, lse = _run(q, cache, t, cu, lens, 0.1, True)
    cref.check_attention(q, cache, t, cu, lens, 0.1, True, o.cpu(), lse.cpu(), 4)


@pytest.mark.parametrize("dqk,dv,Hkv,G,seqs", [(64, 64, 16, 4, [(1100, 1100)]), (128, 128, 16, 4, [(700, 900), (650, 650)]), (256, 256, 16, 4, [(600, 640)])])
def test_undivided(dqk, dv, Hkv, G, seqs):
    """Rows enough that no keys are divided."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(3, seqs, Hkv, G, dqk, dv, 4, 64, BF)
    c = cref.on_gpu(cache)
    assert A.attn_cache_chunk_workspace_bytes(c, len(seqs), q.shape[0], Hkv * G, t.shape[1]) == 256
    o, lse = _run(q, c, t, cu, lens, dqk ** -0.5, True)
    cref.check_attention(q, cache, t, cu, lens, dqk ** -0.5, True, o.cpu(), lse.cpu(), 4)


@pytest.mark.parametrize("dqk,dv,bits", [(64, 64, 8), (128, 128, 4), (192, 128, 8)])
def test_long_keys_divided(dqk, dv, bits):
    q, cache, t, cu, lens = _case(9, [(17, 9001), (1, 3333)], 2, 4, dqk, dv, bits, 64, HF)
    o, lse = _run(q, cache, t, cu, lens, dqk ** -0.5, True)
    cref.check_attention(q, cache, t, cu, lens, dqk ** -0.5, True, o.cpu(), lse.cpu(), bits)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dqk,dv,bits", [(64, 64, 8), (96, 96, 4), (192, 128, 4), (256, 256, 8)])
def test_few_rows_divided(dqk, dv, bits, causal):
    """Up to 128 rows, whose keys are divided, next to one that has more, one without keys and one without queries."""
    q, cache, t, cu, lens = _case(dqk, [(25, 3000), (17, 1500), (32, 2049), (1, 2500), (33, 1100), (5, 0), (0, 900), (16, 31)], 2, 4, dqk, dv, bits, 32, BF)
    o, lse = _run(q, cache, t, cu, lens, dqk ** -0.5, causal)
    cref.check_attention(q, cache, t, cu, lens, dqk ** -0.5, causal, o.cpu(), lse.cpu(), bits)


def test_many_sequences():
    """More than a wave has lanes, some without queries, some without keys, lengths beyond the table and negative ones."""
    g = cref.gen(5)
    seqs = [(int(a), int(n)) for a, n in zip(torch.randint(0, 9, (150,), generator=g), torch.randint(0, 120, (150,), generator=g))]
    q, cache, t, cu, lens = _case(6, seqs, 2, 2, 64, 64, 4, 16, BF)
    full = int((torch.tensor([n for _, n in seqs])).argmax())
    lens[full] = 10 ** 6                                       # (its pages fill the table's row but for the last one's end)
    lens[(full + 1) % 150] = -5
    lens[full] = lens[full] if seqs[full][1] % 16 == 0 else seqs[full][1]
    for causal in (True, False):
        o, lse = _run(q, cache, t, cu, lens, 0.125, causal)
        cref.check_attention(q, cache, t, cu, lens, 0.125, causal, o.cpu(), lse.cpu(), 4)


def test_lengths_beyond_the_table():
    q, cache, t, cu, lens = _case(8, [(20, 128), (3, 64)], 1, 2, 64, 64, 4, 64, BF)
    want = _run(q, cache, t, cu, lens, 0.125, True)
    got = _run(q, cache, t, cu, torch.tensor([2 ** 31 - 1, 64], dtype=torch.int32), 0.125, True)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_views_padding_and_given_outputs():
    """A slice of a fused projection, rows of no sequence between and behind, outputs of the caller's."""
    import paper_2603_05451_amd as A
    seqs = [(9, 40), (70, 75)]
    q, cache, t, _, lens = _case(4, seqs, 2, 2, 128, 128, 8, 32, BF, pad=30)
    T = q.shape[0]
    cu = torch.tensor([5, 14, 84], dtype=torch.int32)
    wide = torch.zeros(T, 7, 136, dtype=BF, device="cuda")
    wide[:, 2:6, :128] = q.cuda()
    o = torch.full((4, T, 128), 7.0, dtype=BF, device="cuda").transpose(0, 1)
    lse = torch.full((4, T), 7.0, device="cuda")
    c = cref.on_gpu(cache)
    ws = torch.empty(A.attn_cache_chunk_workspace_bytes(c, 2, T, 4, t.shape[1]), dtype=torch.uint8, device="cuda")
    r = A.attn_cache_chunk_fwd(wide[:, 2:6, :128], c, t.cuda(), cu.cuda(), lens.cuda(), 0.1, True, o=o, lse=lse, workspace=ws)
    assert r[0] is o and r[1] is lse
    cref.check_attention(q, cache, t, cu, lens, 0.1, True, o.cpu(), lse.cpu(), 8)
    free = [*range(5), *range(84, T)]
    assert (o[free] == 7).all() and (lse[:, free] == 7).all()
    again = _run(q, c, t, cu, lens, 0.1, True)
    assert torch.equal(again[0][5:84], o[5:84]) and torch.equal(again[1][:, 5:84], lse[:, 5:84])


def test_boundaries_out_of_order():
    """Sequences whose boundaries do not ascend, or lie outside, have no queries; the others are as they would be alone."""
    seqs = [(10, 50), (10, 60), (10, 70)]
    q, cache, t, cu, lens = _case(2, seqs, 1, 4, 64, 64, 4, 16, BF)
    want = _run(q, cache, t, cu, lens, 0.125, True)
    o, lse = torch.full_like(want[0], 3.0), torch.full_like(want[1], 3.0)
    bad = torch.tensor([0, 10, 2 ** 31 - 1, 30], dtype=torch.int32)
    _run(q, cache, t, bad, lens, 0.125, True, o=o, lse=lse)
    assert torch.equal(o[:10], want[0][:10]) and torch.equal(lse[:, :10], want[1][:, :10]) and (o[10:] == 3).all() and (lse[:, 10:] == 3).all()
    bad = torch.tensor([-7, 0, 10, 5], dtype=torch.int32)
    _run(q, cache, t, bad, lens, 0.125, True, o=o, lse=lse)
    assert (o[10:] == 3).all()


@pytest.mark.parametrize("fill", [0x7f, 0xff, 0x01, 0x00])
def test_sequences_that_share_queries(fill):
    """More work than T queries can have: some of it has no blocks.  What the workspace held before is not taken for where parts are, and only rows of
    the sequences are written."""
    import paper_2603_05451_amd as A
    q, cache, t, _, _ = _case(9, [(40, 4000)], 2, 4, 64, 64, 4, 64, BF, pad=40)
    cu = torch.tensor([0, 40] * 400 + [40, 70], dtype=torch.int32)          # every second sequence has none, for its boundaries descend
    B = cu.numel() - 1
    t, lens = t[:1].expand(B, -1).contiguous(), torch.full((B,), 4000, dtype=torch.int32)
    n = A.attn_cache_chunk_workspace_bytes(cref.on_gpu(cache), B, 80, 8, t.shape[1])
    ws = torch.full((n + 512,), fill, dtype=torch.uint8, device="cuda")
    o, lse = torch.full((80, 8, 64), 3.0, dtype=BF, device="cuda"), torch.full((8, 80), 3.0, device="cuda")
    _run(q, cache, t, cu, lens, 0.125, True, o=o, lse=lse, workspace=ws[:n])
    assert n > 256 and (ws[n:] == fill).all() and (o[70:] == 3).all() and (lse[:, 70:] == 3).all()


@pytest.mark.parametrize("bits,dtype", [(4, BF), (8, BF), (4, HF), (8, HF)])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (256, 256)])
def test_numbers_that_are_not_finite(dqk, dv, bits, dtype):
    """NaN in values reaches the queries that see them, in their channels, and no others; in keys the queries that see them; behind the last key and on
    pages that are not there (but under no visible key) none."""
    seqs = [(80, 100), (40, 200)]
    q, cache, t, cu, lens = _case(11, seqs, 2, 2, dqk, dv, bits, 16, dtype)
    page = lambda b, j: (int(t[b, j // 16]), j % 16)
    clean = [x.clone() for x in cache]
    kill = [(0, 20, 1, 1), (0, 50, 0, 0), (0, 99, 1, 0), (1, 170, 0, 1)]           # sequence, key, head, block of 32 channels
    for b, j, h, blk in kill:
        p, at = page(b, j)
        cache[3][p, h, at, blk] = 255
    for b, n in enumerate((100, 200)):                                             # the rest of the last pages
        for j in range(n, -(-n // 16) * 16):
            p, at = page(b, j)
            for x in cache:
                x[p, :, at] = 255
    o, lse = (x.cpu() for x in _run(q, cache, t, cu, lens, dqk ** -0.5, True))
    wo, wl = (x.cpu() for x in _run(q, clean, t, cu, lens, dqk ** -0.5, True))
    assert torch.equal(lse, wl)
    hit = torch.zeros(120, 4, dv, dtype=torch.bool)
    for b, j, h, blk in kill:
        nq, n = seqs[b]
        first = max(0, j - (n - nq))                                               # the first query that sees key j
        hit[int(cu[b]) + first:int(cu[b + 1]), 2 * h:2 * h + 2, 32 * blk:32 * blk + 32] = True
    assert (~torch.isfinite(o))[hit].all() and torch.equal(o[~hit], wo[~hit])
    # a key
    cache = [x.clone() for x in clean]
    p, at = page(0, 60)
    cache[1][p, 1, at, 0] = 255
    o, lse = (x.cpu() for x in _run(q, cache, t, cu, lens, dqk ** -0.5, True))
    hit = torch.zeros(120, 4, dtype=torch.bool)
    hit[40:80, 2:] = True
    assert torch.isnan(o[hit]).all() and torch.isnan(lse.T[hit]).all() and torch.equal(o[~hit], wo[~hit]) and torch.equal(lse.T[~hit], wl.T[~hit])


def test_values_that_fp16_cannot_hold():
    """4 * 2^14 and more are infinite as fp16 numbers, and fine as bf16 ones."""
    q, cache, t, cu, lens = _case(13, [(50, 50)], 1, 1, 64, 64, 8, 16, HF)
    p, at = int(t[0, 30 // 16]), 30 % 16
    cache[2][p, 0, at], cache[3][p, 0, at] = 0x70, 127 + 9                          # 128 * 2^9 = 2^16
    o, _ = _run(q, cache, t, cu, lens, 0.125, True)
    assert torch.isfinite(o[:30]).all() and torch.isposinf(o[30:]).all()
    o, lse = _run(q.to(BF), cache, t, cu, lens, 0.125, True)
    cref.check_attention(q.to(BF), cache, t, cu, lens, 0.125, True, o.cpu(), lse.cpu(), 8)


def test_pages_outside_the_cache():
    """Rows that see a key of such a page are NaN; others are as without it."""
    q, cache, t, cu, lens = _case(17, [(60, 60), (5, 90)], 2, 1, 128, 128, 4, 16, BF)
    want = [x.cpu() for x in _run(q, cache, t, cu, lens, 0.1, True)]
    for bad in (-1, cache[0].shape[0], 2 ** 31 - 1, -(2 ** 31)):
        u = t.clone()
        u[0, 2] = bad                                                              # keys 32 ... 47
        o, lse = (x.cpu() for x in _run(q, cache, u, cu, lens, 0.1, True))
        assert torch.isnan(o[32:60]).all() and torch.isnan(lse[:, 32:60]).all()
        assert torch.equal(o[:32], want[0][:32]) and torch.equal(o[60:], want[0][60:]) and torch.equal(lse[:, 60:], want[1][:, 60:])


def test_like_attention_of_few_queries():
    """A batch of equal chunks: attn_cache_fwd's results up to rounding (both are checked against 64 bits elsewhere)."""
    import paper_2603_05451_amd as A
    q, cache, t, cu, lens = _case(19, [(4, 500)] * 6, 2, 4, 128, 128, 4, 64, BF)
    c = cref.on_gpu(cache)
    o, lse = _run(q, c, t, cu, lens, 0.09, True)
    po, pl = A.attn_cache_fwd(q.cuda().view(6, 4, 8, 128), c, t.cuda(), lens.cuda(), 0.09, True)
    assert float((o.view_as(po).float() - po.float()).norm() / po.float().norm()) < 2 * 2.0 ** -8
    assert float((lse.view(8, 6, 4).transpose(0, 1) - pl).abs().max()) < 1e-4


def test_again_on_a_stream_and_in_a_graph():
    """The same bits every time: twice, on another stream, captured and replayed with other boundaries, lengths, pages and queries."""
    import paper_2603_05451_amd as A
    a = _case(21, [(30, 400), (1, 900), (77, 77)], 2, 2, 128, 128, 4, 64, BF, spare=30)
    b = _case(22, [(100, 150), (0, 700), (8, 850)], 2, 2, 128, 128, 4, 64, BF, spare=30)
    c = cref.on_gpu(a[1])
    width = max(a[2].shape[1], b[2].shape[1])
    pad = lambda t: torch.nn.functional.pad(t, (0, width - t.shape[1])) % a[1][0].shape[0]
    T = max(a[0].shape[0], b[0].shape[0])
    state = {"q": torch.zeros(T, 4, 128, dtype=BF, device="cuda"), "t": torch.zeros(3, width, dtype=torch.int32, device="cuda"),
             "cu": torch.zeros(4, dtype=torch.int32, device="cuda"), "lens": torch.zeros(3, dtype=torch.int32, device="cuda"),
             "o": torch.zeros(T, 4, 128, dtype=BF, device="cuda"), "lse": torch.zeros(4, T, device="cuda")}
    ws = torch.empty(A.attn_cache_chunk_workspace_bytes(c, 3, T, 4, width), dtype=torch.uint8, device="cuda")

    def put(x):
        state["q"].zero_()
        state["q"][:x[0].shape[0]] = x[0].cuda()
        for name, y in (("t", pad(x[2])), ("cu", x[3]), ("lens", x[4])):
            state[name].copy_(y.cuda())
        state["o"].fill_(5.0)
        state["lse"].fill_(5.0)

    def call():
        A.attn_cache_chunk_fwd(state["q"], c, state["t"], state["cu"], state["lens"], 0.1, True, o=state["o"], lse=state["lse"], workspace=ws)

    def result(x):
        put(x)
        call()
        return state["o"].clone(), state["lse"].clone()
    want = [result(a), result(b)]
    assert all(torch.equal(x, y) for x, y in zip(want[0], result(a)))
    side = torch.cuda.Stream()
    put(b)
    torch.cuda.synchronize()
    A.attn_cache_chunk_fwd(state["q"], c, state["t"], state["cu"], state["lens"], 0.1, True, o=state["o"], lse=state["lse"], workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(state["o"], want[1][0]) and torch.equal(state["lse"], want[1][1])
    graph = torch.cuda.CUDAGraph()
    put(a)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for x, w in ((b, want[1]), (a, want[0]), (b, want[1]), (a, want[0])):
        put(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(state["o"], w[0]) and torch.equal(state["lse"], w[1])
