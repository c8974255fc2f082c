"""GPU tests of the quantised cache: attn_cache_write and attn_cache_read, which are exact (codes, scales and values are compared for
equality), and attn_cache_fwd, against definitions in 64 bits on what the cache holds.

Tolerance of the attention, per element: the output's rounding, half a step (eps/2) of the result; P's rounding to the element type,
eps/2 of sum_j P_j |V_j|; and fp32: a score, a sum of d products, is off by at most (d + 8) 2^-24 of its terms' sizes, which is what P is
off relatively (and again through the row sum), exp2, the merges and the row sum's n terms add n / 32 + 64 steps of 2^-24 (a lane sums every
32nd key).  LSE: the score's error, the row sum's, and 2^-23 of itself."""
import math

import pytest
import torch

import ops_reference as ref

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
DIMS = [(64, 64), (96, 96), (128, 128), (192, 128), (256, 256)]


def _gen(seed):
    return torch.Generator("cpu").manual_seed(seed)


def _random_cache(gen, pages, page, Hkv, dqk, dv, bits):
    """A cache of random finite codes and scales about 1, on the CPU."""
    out = []
    for d in (dqk, dv):
        raw = torch.randint(0, 256, (pages, Hkv, page, d * bits // 8), generator=gen, dtype=torch.uint8)
        if bits == 8:
            raw = torch.where((raw & 0x7f) > 0x47, raw & 0xb7, raw)          # |code| <= 16 ...
        sc = torch.randint(123, 127, (pages, Hkv, page, d // 32), generator=gen).to(torch.uint8) - (2 if bits == 8 else 0)
        out += [raw, sc]
    return out


def _on_gpu(cache):
    import paper_2603_05451_amd as A
    return A.AttnCache(*(t.cuda() for t in cache))


# ---------------------------------------------------------------------------------------------- writing and reading

def _specials(x, dtype):
    """Blocks with ties, zeros, infinities, NaN, the smallest and the largest numbers among the rows of x [T, H, d]."""
    lim = torch.finfo(dtype)
    x[0, 0, :32] = 0
    x[0, 0, 32:64] = -0.0
    if x.shape[0] > 4:
        x[1, 0, 3], x[1, 0, 40] = math.inf, -math.inf
        x[2, 0, 5] = math.nan
        x[3, 0, :32] = torch.tensor([6, 0.25, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, 4.5, 5.5, 2.25, 0.5, 0, -0.75] * 2).to(dtype)
        x[3, 0, 32:64] = torch.tensor([448, 464, 1.0625, 1.1875, 17, 19, 2 ** -10, 3 * 2 ** -10] * 4).to(dtype)
        x[4, 0, :32] = (torch.arange(32) * lim.smallest_normal / 16).to(dtype)
        x[4, 0, 32:64] = (torch.linspace(-1, 1, 32) * lim.max).to(dtype)
    return x


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("dtype,T,Hkv,page", [(BF, 1, 1, 16), (BF, 77, 3, 64), (HF, 130, 2, 32)])
def test_write_and_read(bits, dqk, dv, dtype, T, Hkv, page):
    import paper_2603_05451_amd as A
    gen = _gen(T + bits)
    pages = T // page + 3
    before = _random_cache(gen, pages, page, Hkv, dqk, dv, bits)
    cache = _on_gpu(before)
    big = torch.exp(3 * torch.randn(T, 1, 1, generator=gen))
    k, v = (_specials((torch.randn(T, Hkv, d, generator=gen) * big).to(dtype), dtype) for d in (dqk, dv))
    slots = torch.randperm(pages * page, generator=gen)[:T].int()
    if T > 20:
        slots[5], slots[11], slots[12], slots[13] = -1, pages * page, 2 ** 31 - 1, -(2 ** 31)
    buf = torch.zeros(T, Hkv + 2, dqk + 8, dtype=dtype, device="cuda")                 # keys: a view; values: contiguous
    buf[:, 1:1 + Hkv, :dqk] = k.cuda()
    assert A.attn_cache_write(buf[:, 1:1 + Hkv, :dqk], v.cuda(), slots.cuda(), cache) is None
    there = (slots >= 0) & (slots < pages * page)
    at = slots[there].long()
    want = [t.clone() for t in before]
    for x, i in ((k, 0), (v, 2)):
        code, scale = ref.quantise(x[there], bits)
        want[i][at // page, :, at % page] = ref.pack(code, bits)
        want[i + 1][at // page, :, at % page] = scale.to(torch.uint8)
    for got, w, name in zip(cache, want, cache._fields):
        assert torch.equal(got.cpu(), w), name
    # back: these slots, and others, some twice, some nowhere
    ask = torch.cat((slots, torch.randint(-3, pages * page + 3, (41,), generator=gen).int(), slots[:1]))
    out = A.attn_cache_read(ask.cuda(), cache, dtype)
    there = (ask >= 0) & (ask < pages * page)
    for got, i, d in zip(out, (0, 2), (dqk, dv)):
        full = torch.zeros(len(ask), Hkv, d, dtype=torch.float64)
        full[there] = ref.rows(want[i], want[i + 1], ask[there], bits)
        full = full.to(torch.float32).to(dtype)
        assert got.shape == full.shape and got.is_contiguous()
        assert torch.equal(torch.nan_to_num(got.cpu(), nan=77.0), torch.nan_to_num(full, nan=77.0))
    again = [torch.full_like(t, 3.0) for t in out]
    assert A.attn_cache_read(ask.cuda(), cache, dtype, k=again[0], v=again[1])[0] is again[0]
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(again, out))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_every_code_reads_back(dtype):
    """All codes under all scales: what a cache may hold, bit for bit as a conversion from the exact number."""
    import paper_2603_05451_amd as A
    for bits in (4, 8):
        codes = torch.arange(256, dtype=torch.uint8).repeat(32)[:16 * 64 * bits // 8].view(1, 1, 16, -1).repeat(256, 1, 1, 1)
        codes = torch.cat([codes[:, :, :, :], codes.flip(-1)], dim=2)                # page 32
        scale = torch.arange(256, dtype=torch.uint8).view(256, 1, 1, 1).repeat(1, 1, 32, 2)
        cache = A.AttnCache(*(t.contiguous().cuda() for t in (codes, scale, codes, scale)))
        slots = torch.arange(256 * 32, dtype=torch.int32)
        k, v = A.attn_cache_read(slots.cuda(), cache, dtype)
        want = ref.rows(codes, scale, slots, bits)
        # (exact numbers: to fp32 first, which holds all but subnormals of 2^-127 blocks exactly, and those are below every half step of bf16)
        want = torch.nan_to_num(want.to(torch.float32).to(dtype), nan=77.0, posinf=math.inf, neginf=-math.inf)
        assert torch.equal(torch.nan_to_num(k.cpu(), nan=77.0, posinf=math.inf, neginf=-math.inf), want) and torch.equal(k.view(torch.int16), v.view(torch.int16))


# ---------------------------------------------------------------------------------------------- attention

def _table(gen, lens, page, pages, width=None):
    """Distinct pages for every sequence, in no order; nonsense behind the last one."""
    need = [max(0, -(-n // page)) for n in lens]
    width = width or max(1, max(need))
    order = torch.randperm(pages, generator=gen)
    table = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(lens), width), generator=gen).int()
    i = 0
    for b, n in enumerate(need):
        table[b, :n] = order[i:i + n]
        i += n
    return table


def _check(q, cache, table, lens, scale, causal, o, lse, bits, only=None):
    """q, cache, table, lens, o, lse on the CPU."""
    B, Nq, H, d = q.shape
    page, dtype = cache[0].shape[2], q.dtype
    half = ref.HALF[dtype]
    for b in range(B) if only is None else only:
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        j = torch.arange(n)
        slots = table[b, j // page].long() * page + j % page
        k, v = (ref.rows(cache[i], cache[i + 1], slots, bits) for i in (0, 2))
        limits = [n - Nq + i if causal else n - 1 for i in range(Nq)]
        wo, wl, size, terms = ref.attend(q[b].double(), k, v, scale, limits)
        seen = torch.isfinite(wl)
        assert torch.equal(torch.isneginf(lse[b]), ~seen)
        steps = (d + 8) * terms + n / 32 + 64
        off = (lse[b].double() - wl)[seen].abs() - (steps[seen] * 2.0 ** -24 + 2.0 ** -23 * wl[seen].abs())
        assert off.numel() == 0 or off.max() <= 0, off.max()
        bound = half * wo.abs() + ref.TINY[dtype] + (half + 2 * steps.T[..., None] * 2.0 ** -24) * (size + wo.abs())
        worst = ((o[b].double() - wo).abs() - bound).max()
        assert worst <= 0, (b, n, worst)
        assert (o[b][~seen.T] == 0).all()


def _run(seed, lens, Nq, H, Hkv, dqk, dv, bits, page, dtype, causal, view=False, width=None):
    import paper_2603_05451_amd as A
    gen = _gen(seed)
    pages = sum(-(-max(n, 0) // page) for n in lens) + 2
    cache = _random_cache(gen, pages, page, Hkv, dqk, dv, bits)
    table = _table(gen, lens, page, pages, width)
    lens = torch.tensor(lens, dtype=torch.int32)
    q = torch.randn(len(lens), Nq, H, dqk, generator=gen).to(dtype)
    qg, out = q.cuda(), None
    if view:
        qg = qg.transpose(1, 2).contiguous().transpose(1, 2)
        out = torch.full((len(lens), H, Nq, dv + 16), 5.0, dtype=dtype, device="cuda")[..., :dv].transpose(1, 2)
    o, lse = A.attn_cache_fwd(qg, _on_gpu(cache), table.cuda(), lens.cuda(), dqk ** -0.5, causal, o=out)
    torch.cuda.synchronize()
    assert out is None or o is out
    _check(q, cache, table, lens, dqk ** -0.5, causal, o.cpu(), lse.cpu(), bits)
    if view:
        assert (out.transpose(1, 2).as_strided((len(lens), H, Nq, 16), (H * Nq * (dv + 16), Nq * (dv + 16), dv + 16, 1), dv) == 5).all()


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("dtype,H,Hkv,page", [(BF, 4, 1, 16), (HF, 6, 2, 64)])
def test_single_tokens_at_the_edges(bits, dqk, dv, dtype, H, Hkv, page):
    _run(1, EDGES, 1, H, Hkv, dqk, dv, bits, page, dtype, True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("Nq,H,Hkv,causal", [(3, 6, 2, True), (5, 4, 1, True), (4, 8, 1, False)])
def test_several_queries(bits, dqk, dv, Nq, H, Hkv, causal):
    """9, 20 and 32 rows a group: one and two row blocks; rows before the first key."""
    _run(2, [0, 1, 2, 3, 4, 5, 31, 33, 36, 100, 259, 320], Nq, H, Hkv, dqk, dv, bits, 32, BF if causal else HF, causal, view=Nq == 5)


@pytest.mark.parametrize("Nq,H,Hkv,page", [(1, 48, 1, 16), (7, 16, 2, 128), (40, 2, 2, 64), (1, 1, 1, 256)])
def test_many_rows(Nq, H, Hkv, page):
    """48, 56 and 40 rows: several groups of rows; one row."""
    _run(3, [70, 0, 39, 41, 300], Nq, H, Hkv, 128, 128, 4, page, BF, True)


@pytest.mark.parametrize("dtype,lens,H,Hkv,bits", [
    (BF, [9001], 4, 1, 4), (BF, [4000, 3, 0, 257, 1025, 2048], 8, 2, 4), (HF, [5000, 1, 600], 2, 2, 8),
    (BF, [3000] * 3 + [0, 1, 700] * 40, 2, 1, 4)])
def test_divided_keys(dtype, lens, H, Hkv, bits):
    """Sequences in several chunks beside short and empty ones; more sequences than lanes."""
    _run(4, lens, 1, H, Hkv, 64, 64, bits, 64, dtype, True)


@pytest.mark.parametrize("dqk,dv,bits,B,Nq,H,Hkv,dtype", [
    (64, 64, 4, 600, 1, 4, 2, BF), (64, 64, 8, 530, 3, 12, 2, HF), (96, 96, 4, 400, 1, 2, 2, HF), (96, 96, 8, 270, 5, 8, 2, BF), (128, 128, 4, 400, 1, 2, 2, BF),
    (128, 128, 8, 260, 9, 4, 2, HF), (192, 128, 4, 300, 1, 2, 2, BF), (192, 128, 8, 130, 9, 4, 2, BF), (256, 256, 4, 300, 1, 2, 2, HF), (256, 256, 8, 130, 9, 4, 2, BF)])
def test_more_sequences_than_blocks(dqk, dv, bits, B, Nq, H, Hkv, dtype):
    """A wave per (sequence, KV head): short and empty sequences, a few of several chunks among them, more than 512 of them."""
    gen = _gen(B + dqk)
    lens = [int(x) for x in torch.randint(0, 70, (B,), generator=gen)]
    for b in (0, B // 2, B - 1):
        lens[b] = 1300 + b
    _run(B, lens, Nq, H, Hkv, dqk, dv, bits, 32, dtype, True, view=bits == 8)


def test_another_device_than_the_current_one(monkeypatch):
    import paper_2603_05451_amd as A
    q, f = torch.zeros(1, 8, 4, 64, dtype=BF, device="cuda"), A.attn_rope_freqs(64)
    c = A.attn_cache_new(4, 16, 2, 64, 64)
    i = torch.zeros(8, dtype=torch.int32, device="cuda")
    A.lib()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)

    class Left:                                 # (the native part asks for the device in its own way, and leaves such calls alone)
        def __getattr__(self, name):
            return lambda *a: None
    monkeypatch.setattr(A, "_native", Left())
    for call in (lambda: A.attn_rope_fwd(q, None, f), lambda: A.attn_rope_bwd(q, None, f), lambda: A.attn_cache_read(i, c, BF),
                 lambda: A.attn_cache_write(q[0, :, :2], q[0, :, :2], i, c), lambda: A.attn_cache_fwd(q, c, i.view(1, 8), i[:1], 0.1, True),
                 lambda: A.attn_rope_fwd(q, None, f, stream=torch.cuda.current_stream(0))):
        with pytest.raises(ValueError, match="device"):
            call()


def test_wide_table_and_lengths_beyond_it():
    """A table with room for more keys than there are, and lengths that it has no room for or that are negative."""
    import paper_2603_05451_amd as A
    _run(5, [100, 0, 33], 2, 4, 2, 128, 128, 4, 16, BF, True, width=5000)
    gen = _gen(6)
    cache = _random_cache(gen, 12, 16, 1, 64, 64, 4)
    table = torch.randperm(12, generator=gen).int().view(3, 4)
    q = torch.randn(3, 1, 2, 64, generator=gen).to(BF)
    for lens in ([65, 2 ** 31 - 1, 64], [-1, -(2 ** 31), 5]):
        lens = torch.tensor(lens, dtype=torch.int32)
        o, lse = A.attn_cache_fwd(q.cuda(), _on_gpu(cache), table.cuda(), lens.cuda(), 0.125, True)
        _check(q, cache, table, lens, 0.125, True, o.cpu(), lse.cpu(), 4)


@pytest.mark.parametrize("bits", [4, 8])
def test_what_lies_behind_the_last_key(bits):
    """NaN in the rest of the last page and in pages that are not listed reaches nothing."""
    import paper_2603_05451_amd as A
    gen = _gen(7)
    lens = [5, 16, 17, 40, 0, 63, 200]
    cache = _random_cache(gen, 40, 16, 2, 128, 128, bits)
    table = _table(gen, lens, 16, 40)
    held = torch.zeros(40 * 16, dtype=torch.bool)
    for b, n in enumerate(lens):
        j = torch.arange(n)
        held[table[b, j // 16].long() * 16 + j % 16] = True
    free = ~held.view(40, 16)
    for t, x in zip(cache, (0xff, 255, 0xff, 255)):
        t.permute(0, 2, 1, 3)[free] = x
    q, lens = torch.randn(7, 3, 4, 128, generator=gen).to(BF), torch.tensor(lens, dtype=torch.int32)
    o, lse = A.attn_cache_fwd(q.cuda(), _on_gpu(cache), table.cuda(), lens.cuda(), 0.1, True)
    _check(q, cache, table, lens, 0.1, True, o.cpu(), lse.cpu(), bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (96, 96), (192, 128)])
def test_numbers_that_are_none_reach_who_sees_them(bits, dqk, dv):
    """A NaN block of the last-but-one key or value: queries before it are untouched, the others have it where it belongs."""
    import paper_2603_05451_amd as A
    gen = _gen(8)
    n, Nq, H = 70, 4, 4
    cache = _random_cache(gen, 5, 16, 2, dqk, dv, bits)
    table = torch.randperm(5, generator=gen).int().view(1, 5)
    q, lens = torch.randn(1, Nq, H, dqk, generator=gen).to(BF), torch.tensor([n], dtype=torch.int32)
    run = lambda c: [t.cpu() for t in A.attn_cache_fwd(q.cuda(), _on_gpu(c), table.cuda(), lens.cuda(), 0.1, True)]
    o, lse = run(cache)
    at = (int(table[0, (n - 2) // 16]), 0, (n - 2) % 16)                 # KV head 0: query heads 0 and 1; queries 2 and 3 see it
    bad = [t.clone() for t in cache]
    bad[3][at][1] = 255                                                  # channels 32 ... 63 of the value
    bo, blse = run(bad)
    assert torch.equal(blse, lse) and torch.isnan(bo[0, 2:, :2, 32:64].float()).all()
    bo[0, 2:, :2, 32:64] = o[0, 2:, :2, 32:64]
    assert torch.equal(bo, o)
    bad = [t.clone() for t in cache]
    bad[1][at][0] = 255
    bo, blse = run(bad)
    assert torch.isnan(bo[0, 2:, :2].float()).all() and torch.isnan(blse[0, :2, 2:]).all()
    bo[0, 2:, :2], blse[0, :2, 2:] = o[0, 2:, :2], lse[0, :2, 2:]
    assert torch.equal(bo, o) and torch.equal(blse, lse)


def test_pages_outside_the_cache():
    """Rows that see a key on such a page are NaN, the others are served."""
    import paper_2603_05451_amd as A
    gen = _gen(9)
    cache = _random_cache(gen, 8, 32, 1, 128, 128, 4)
    q, lens = torch.randn(4, 1, 2, 128, generator=gen).to(BF), torch.tensor([64, 64, 40, 32], dtype=torch.int32)
    table = torch.tensor([[0, 1], [2, 8], [-1, 3], [4, 2 ** 31 - 1]], dtype=torch.int32)
    o, lse = (t.cpu() for t in A.attn_cache_fwd(q.cuda(), _on_gpu(cache), table.cuda(), lens.cuda(), 0.1, True))
    assert torch.isnan(o[1:3].float()).all() and torch.isnan(lse[1:3]).all()
    _check(q, cache, table, lens, 0.1, True, o, lse, 4, only=[0, 3])


def test_offsets_beyond_32_bits():
    """The last pages of a cache whose codes take more than 4 GiB."""
    import paper_2603_05451_amd as A
    pages, page, Hkv, d = 33000, 64, 16, 128
    cache = A.attn_cache_new(pages, page, Hkv, d, d, bits=8)
    assert cache.k.numel() > 2 ** 32
    gen = _gen(10)
    k, v = (torch.randn(150, Hkv, d, generator=gen).to(BF) for _ in range(2))
    table = torch.tensor([[pages - 1, 1, pages - 2]], dtype=torch.int32)
    j = torch.arange(150)
    slots = (table[0, j // page].long() * page + j % page).int()
    A.attn_cache_write(k.cuda(), v.cuda(), slots.cuda(), cache)
    back = A.attn_cache_read(slots.cuda(), cache, BF)
    want = [ref.values(*ref.quantise(x, 8), 8) for x in (k, v)]
    assert all(torch.equal(g.double().cpu(), w) for g, w in zip(back, want))
    assert int(cache.k[:1].max()) == 0 and int(cache.k[pages - 3].max()) == 0
    q = torch.randn(1, 1, Hkv, d, generator=gen).to(BF)
    o, lse = A.attn_cache_fwd(q.cuda(), cache, table.cuda(), torch.tensor([150], dtype=torch.int32).cuda(), 0.1, True)
    wo, wl, size, terms = ref.attend(q[0].double(), *want, 0.1, [149])
    assert (lse[0].cpu().double() - wl).abs().max() <= ((d + 8) * terms.max() + 100) * 2.0 ** -24 + 2.0 ** -23 * wl.abs().max()
    assert ((o[0].cpu().double() - wo).abs() <= 2.0 ** -7 * (size + wo.abs())).all()


def test_refusals_of_tensors():
    import paper_2603_05451_amd as A
    c = A.attn_cache_new(4, 16, 2, 64, 64)
    q, table, lens = torch.zeros(3, 1, 4, 64, dtype=BF, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    k, slots = torch.zeros(5, 2, 64, dtype=BF, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda")
    other = A.attn_cache_new(4, 16, 2, 128, 128)
    bad = [lambda: A.attn_cache_fwd(q.float(), c, table, lens, 0.1, True), lambda: A.attn_cache_fwd(q[..., :32], c, table, lens, 0.1, True),
           lambda: A.attn_cache_fwd(q, other, table, lens, 0.1, True), lambda: A.attn_cache_fwd(q[:, 0], c, table, lens, 0.1, True),
           lambda: A.attn_cache_fwd(q, c, table.long(), lens, 0.1, True), lambda: A.attn_cache_fwd(q, c, table[:2], lens, 0.1, True),
           lambda: A.attn_cache_fwd(q, c, table[0], lens, 0.1, True), lambda: A.attn_cache_fwd(q, c, table, lens[:2], 0.1, True),
           lambda: A.attn_cache_fwd(q, c, table.cpu(), lens, 0.1, True), lambda: A.attn_cache_fwd(q, c._replace(v=c.v.int()), table, lens, 0.1, True),
           lambda: A.attn_cache_fwd(q, c._replace(k=c.k[:3]), table, lens, 0.1, True), lambda: A.attn_cache_fwd(q, c._replace(v_scale=other.v_scale), table, lens, 0.1, True),
           lambda: A.attn_cache_fwd(q, c._replace(k=c.k[..., :16].contiguous()), table, lens, 0.1, True), lambda: A.attn_cache_fwd(q, c._replace(k=c.k.cpu()), table, lens, 0.1, True),
           lambda: A.attn_cache_fwd(q, c, table, lens, 0.1, True, o=q.half()), lambda: A.attn_cache_fwd(q, c, table, lens, 0.1, True, lse=q),
           lambda: A.attn_cache_fwd(q, c, table, lens, 0.1, True, workspace=q),
           lambda: A.attn_cache_write(k, k.half(), slots, c), lambda: A.attn_cache_write(k, k[:4], slots, c), lambda: A.attn_cache_write(k, k, slots[:4], c),
           lambda: A.attn_cache_write(k, k, slots.long(), c), lambda: A.attn_cache_write(k[..., :32], k, slots, c), lambda: A.attn_cache_write(k[None], k[None], slots, c),
           lambda: A.attn_cache_read(slots, c, torch.float32), lambda: A.attn_cache_read(slots[None], c, BF), lambda: A.attn_cache_read(slots, c, BF, k=k, v=k.half()),
           lambda: A.attn_cache_read(slots, c, BF, k=k[:4])]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            assert False, i
    for f in (lambda: A.attn_cache_fwd(q, c, table, lens, 0.0, True), lambda: A.attn_cache_fwd(q[:, :, :3], c, table, lens, 0.1, True),
              lambda: A.attn_cache_fwd(q, c, table, lens, 0.1, True, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda")),
              lambda: A.attn_cache_write(k[:0], k[:0], slots[:0], c), lambda: A.attn_cache_read(slots, A.attn_cache_new(4, 24, 2, 64, 64), BF)):
        with pytest.raises(A.AttnError):
            f()
