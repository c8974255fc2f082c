"""CPU checks of the rotary and cache calls: what the C ABI and the Python functions refuse, the rules that share the work out, and
the tests' own definitions against finite differences."""
import ctypes
import math
import os
import random
import subprocess

import pytest
import torch

import ops_reference as ref

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_05451_amd", "csrc")
P, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    import paper_2603_05451_amd as A
    if not os.path.exists(A.LIB_PATH):
        from paper_2603_05451_amd import build
        build.build_library()
    return A.lib()


def _rope(**over):
    import paper_2603_05451_amd as A
    return A.AttnRope(**{**dict(freqs=0x1000, positions=None, positions_batch=0, rot=64, offset=0, interleaved=0, amplitude=1.0, norm=0,
                                eps=0.0, q_weight=None, k_weight=None), **over})


def _st(*s):
    import paper_2603_05451_amd as A
    return ctypes.byref(A.AttnStrides(*s))


def test_rope_refusals(L):
    import paper_2603_05451_amd as A
    s = _st(10 * 4 * 64, 4 * 64, 64)

    def fwd(r=None, dtype=0, q=P, k=P, qo=P, ko=P, sq=s, sk=s, sqo=s, sko=s, B=2, N=10, H=4, Hkv=4, d=64):
        r = ctypes.byref(_rope() if r is None else r)
        return L.attn_rope_fwd(dtype, r, q, sq, k, sk, qo, sqo, ko, sko, B, N, H, Hkv, d, None)
    bad = [dict(q=None), dict(qo=None), dict(ko=None), dict(k=None), dict(q=ODD), dict(ko=ODD), dict(sq=None), dict(sko=None), dict(B=0),
           dict(N=0), dict(N=-1), dict(H=0), dict(Hkv=0), dict(sq=_st(0, 256, 64)), dict(sk=_st(2560, 260, 64)), dict(sqo=_st(2560, -256, 64)),
           *(dict(r=_rope(**x)) for x in (dict(freqs=None), dict(freqs=0x1002), dict(rot=0), dict(rot=80), dict(rot=64, offset=8), dict(offset=-8),
                                          dict(amplitude=math.nan), dict(amplitude=math.inf), dict(norm=1, eps=-1.0), dict(norm=1, eps=math.nan),
                                          dict(q_weight=0x1000), dict(k_weight=0x1000), dict(norm=1, q_weight=0x1008), dict(positions=0x1001),
                                          dict(positions_batch=-1)))]
    for x in bad:
        assert fwd(**x) == A.ATTN_EINVAL, x
    for x in (dict(dtype=2), dict(d=80), dict(d=32), dict(r=_rope(rot=24)), dict(r=_rope(rot=32, offset=4)), dict(N=1 << 30)):
        assert fwd(**x) == A.ATTN_EUNSUPPORTED, x
    assert L.attn_rope_fwd(0, None, P, s, P, s, P, s, P, s, 2, 10, 4, 4, 64, None) == A.ATTN_EINVAL

    def bwd(r=None, dq=P, dk=P, q=P, k=P, qi=P, ki=P, wq=None, wk=None, ws=P, n=1 << 24):
        r = ctypes.byref(_rope(norm=1, eps=1e-6, q_weight=0x1000, k_weight=0x1000) if r is None else r)
        return L.attn_rope_bwd(0, r, dq, s, dk, s, q, s, k, s, qi, s, ki, s, wq, wk, 2, 10, 4, 4, 64, ws, n, None)
    for x in (dict(dq=None), dict(dk=None), dict(q=None), dict(k=None), dict(qi=None), dict(ki=None), dict(wq=P, ws=None), dict(wk=P, n=256),
              dict(wq=ODD, ws=ctypes.c_void_p(0x1010)), dict(wq=P, r=_rope(norm=1, eps=1e-6)), dict(wk=P, r=_rope())):
        assert bwd(**x) == A.ATTN_EINVAL, x
    assert A.attn_rope_workspace_bytes(2, 10, 4, 4, 64) > 0
    for x in ((0, 10, 4, 4, 64), (2, 10, 4, -1, 64), (2, 10, 4, 4, 80), (2, 1 << 30, 4, 4, 64)):
        assert A.attn_rope_workspace_bytes(*x) == 0


def _cache(**over):
    import paper_2603_05451_amd as A
    return A.AttnCacheLayout(**{**dict(k=0x1000, k_scale=0x1000, v=0x1000, v_scale=0x1000, pages=4, page=32, Hkv=2, d_qk=128, d_v=128, bits=4), **over})


BAD_CACHES = [dict(k=None), dict(v_scale=None), dict(k=0x1008), dict(v=0x1004), dict(pages=0), dict(page=0), dict(Hkv=0)]
FOREIGN_CACHES = [dict(d_qk=64), dict(d_v=80), dict(bits=2), dict(page=8), dict(page=48), dict(page=1 << 17), dict(pages=1 << 27)]


def test_cache_refusals(L):
    import paper_2603_05451_amd as A
    s = _st(0, 2 * 128, 128)

    def write(c=None, dtype=0, k=P, v=P, sk=s, sv=s, slots=P, T=5):
        return L.attn_cache_write(dtype, ctypes.byref(c or _cache()), k, sk, v, sv, slots, T, None)

    def read(c=None, dtype=0, k=P, v=P, slots=P, T=5):
        return L.attn_cache_read(dtype, ctypes.byref(c or _cache()), slots, T, k, v, None)
    for f in (write, read):
        for x in (dict(k=None), dict(v=None), dict(k=ODD), dict(slots=None), dict(slots=ctypes.c_void_p(0x1002)), dict(T=0), dict(T=-3)):
            assert f(**x) == A.ATTN_EINVAL, x
        assert f(dtype=3) == A.ATTN_EUNSUPPORTED
        for x in BAD_CACHES:
            assert f(c=_cache(**x)) == A.ATTN_EINVAL, x
        for x in FOREIGN_CACHES:
            assert f(c=_cache(**x)) == A.ATTN_EUNSUPPORTED, x
    assert write(sk=None) == A.ATTN_EINVAL and write(sv=_st(0, 0, 128)) == A.ATTN_EINVAL and write(sk=_st(0, 260, 128)) == A.ATTN_EINVAL


def test_cache_attention_refusals(L):
    import paper_2603_05451_amd as A
    s = _st(1024, 1024, 128)

    def call(c=None, dtype=0, q=P, sq=s, o=P, so=s, lse=P, table=P, width=4, lens=P, B=3, Nq=1, H=8, scale=0.1, ws=P, n=1 << 30):
        return L.attn_cache_fwd(dtype, ctypes.byref(c or _cache()), q, sq, o, so, lse, table, width, lens, B, Nq, H, scale, 1, ws, n, None)
    for x in (dict(q=None), dict(o=None), dict(lse=None), dict(table=None), dict(lens=None), dict(ws=None), dict(q=ODD), dict(o=ODD),
              dict(lse=ctypes.c_void_p(0x1002)), dict(lens=ctypes.c_void_p(0x1002)), dict(ws=ctypes.c_void_p(0x1010)), dict(width=0), dict(B=0), dict(Nq=0),
              dict(H=0), dict(H=7), dict(scale=0.0), dict(scale=math.nan), dict(sq=None), dict(so=_st(1020, 1024, 128)), dict(width=1000, n=256)):
        assert call(**x) == A.ATTN_EINVAL, x
    for x in (dict(dtype=2), dict(width=1 << 26), dict(width=1 << 21, B=1000), dict(Nq=1 << 22)):
        assert call(**x) == A.ATTN_EUNSUPPORTED, x
    for x in BAD_CACHES:
        assert call(c=_cache(**x)) == A.ATTN_EINVAL, x
    for x in FOREIGN_CACHES:
        assert call(c=_cache(**x)) == A.ATTN_EUNSUPPORTED, x
    size = lambda *a, **c: L.attn_cache_workspace_bytes(ctypes.byref(_cache(**c)), *a)
    assert size(3, 1, 8, 4) == 256 and size(3, 1, 8, 100) > 256 and size(3, 1, 7, 4) == 0 and size(3, 1, 8, 4, bits=3) == 0


def test_launches_within_the_grid(L, rules):
    """Sizes whose blocks would be more than a launch takes are refused, or their rows dealt to fewer blocks."""
    import paper_2603_05451_amd as A
    size = lambda *a, **c: L.attn_cache_workspace_bytes(ctypes.byref(_cache(**c)), *a)
    assert size(65536, 1, 8, 4) > 0 and size(65537, 1, 8, 4) == 0 and size(1 << 20, 1, 64, 1) == 0
    assert size(60000, 1, 512, 64, Hkv=512) == 0 and size(60000, 64, 128, 64) == 0 and size(1, 1 << 20, 16, 1000) > 0
    x = _st(1 << 20, 128, 128)
    s = lambda B, H: L.attn_cache_fwd(0, ctypes.byref(_cache(Hkv=H)), P, x, P, x, P, P, 4, P, B, 1, H, 0.1, 1, P, 1 << 60, None)
    assert s(65537, 2) == A.ATTN_EUNSUPPORTED and s(60000, 1024) == A.ATTN_EUNSUPPORTED
    for tokens, heads in ((1 << 30, 1), (1 << 30, 2), (1023, 1 << 20), (1, 1 << 20)):
        for d in (64, 256):
            blocks, _, shares, _, _ = rules("t_rope", tokens, heads, d, 0)
            assert 0 < blocks <= 1 << 22 and blocks % shares == 0


def test_python_refusals_without_a_gpu():
    import paper_2603_05451_amd as A
    t = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    for f in (lambda: A.attn_rope_fwd(t, None, torch.zeros(32)), lambda: A.attn_rope_bwd(t, None, torch.zeros(32)),
              lambda: A.attn_cache_fwd(t, A.attn_cache_new(2, 16, 2, 64, 64, device="cpu"), torch.zeros(1, 1).int(), torch.zeros(1).int(), 0.1, True),
              lambda: A.attn_cache_read(torch.zeros(3).int(), A.attn_cache_new(2, 16, 2, 64, 64, device="cpu"), torch.bfloat16),
              lambda: A.attn_cache_new(2, 16, 2, 64, 64, bits=3, device="cpu"), lambda: A.attn_rope_freqs(31, device="cpu"),
              lambda: A.attn_rope_freqs(32, factor=0, device="cpu"), lambda: A.attn_rope_freqs(32, original=100, low=3, high=2, device="cpu")):
        with pytest.raises(ValueError):
            f()


def test_frequencies():
    import paper_2603_05451_amd as A
    f = A.attn_rope_freqs(64, base=500000.0, device="cpu").double()
    want = torch.tensor([500000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    assert ((f - want).abs() <= 2.0 ** -24 * want).all()
    assert ((A.attn_rope_freqs(64, factor=4.0, device="cpu").double() - 10000.0 ** (-torch.arange(0, 64, 2).double() / 64) / 4).abs() <= 2.0 ** -24).all()
    g = A.attn_rope_freqs(64, factor=8.0, original=4096, low=1.0, high=32.0, device="cpu").double()
    plain = 10000.0 ** (-torch.arange(0, 64, 2).double() / 64)
    turns = 4096 * plain / (2 * math.pi)
    assert torch.equal(g[turns >= 32], plain[turns >= 32].float().double()) and torch.equal(g[turns <= 1], (plain / 8)[turns <= 1].float().double())
    between = (turns > 1) & (turns < 32)
    assert between.any() and (g[between] < plain[between]).all() and (g[between] > plain[between] / 8).all()


# ---- the definitions that the GPU tests compare with

def test_reference_gradients_against_differences():
    gen = torch.Generator().manual_seed(5)
    normal = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    x, dy, w = normal(2, 3, 2, 64), normal(2, 3, 2, 64), 1 + 0.3 * normal(64)
    pos, f = torch.randint(0, 1000, (2, 3), generator=gen), 100.0 ** (-torch.arange(0, 32, 2).double() / 32)
    for inter in (False, True):
        for eps in (None, 1e-3):
            ww = None if eps is None else w
            loss = lambda x, w: (ref.rope(x, pos, f, 8, inter, 1.25, eps, w)[0] * dy).sum()
            dx, dw, _, _ = ref.rope_bwd(dy, x, pos, f, 8, inter, 1.25, eps, ww)
            h = 1e-5
            for _ in range(3):
                u = normal(*x.shape)
                assert abs((loss(x + h * u, ww) - loss(x - h * u, ww)) / (2 * h) - (dx * u).sum()) < 1e-6 * (dx * u).abs().sum()
                if eps is not None:
                    u = normal(64)
                    assert abs((loss(x, w + h * u) - loss(x, w - h * u)) / (2 * h) - (dw * u).sum()) < 1e-6 * (dw * u).abs().sum()


@pytest.mark.parametrize("bits", [4, 8])
def test_reference_rounding(bits):
    """No element is off by more than half a step of its place, none is cut off, and half the scale would cut one off."""
    gen = torch.Generator().manual_seed(bits)
    x = torch.randn(200, 64, generator=gen).mul(torch.exp(4 * torch.randn(200, 1, generator=gen))).to(torch.bfloat16)
    code, scale = ref.quantise(x, bits)
    v = ref.values(code, scale, bits)
    half = 2.0 ** -2 if bits == 4 else 2.0 ** -4
    small = (2.0 ** (scale.double() - 127)).repeat_interleave(32, -1) * (0.25 if bits == 4 else 2.0 ** -10)
    assert ((v - x.double()).abs() <= torch.maximum(half * x.double().abs(), small)).all()
    top = (x.double().abs().unflatten(-1, (-1, 32)).amax(-1) / 2.0 ** (scale.double() - 127))
    assert (top < 7).all() and (top >= 3.5).all() if bits == 4 else (top <= 464).all() and (top > 232).all()
    assert torch.equal(ref.unpack(ref.pack(code, bits), bits), code)
    tie = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.0] + [0.0] * 23 if bits == 4 else [448.0, 1.0625, 1.1875, 17.0, 2.0 ** -10] + [0.0] * 27)
    got = ref.values(*ref.quantise(tie, bits), bits)
    want = [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0] if bits == 4 else [448.0, 1.0, 1.25, 16.0, 0.0]
    assert got[:len(want)].tolist() == want


# ---- how the work is shared out

SHIM = r"""
#include "ops.h"
using namespace attn;
extern "C" {
void t_cache(int B, int Nq, int H, int Hkv, int d, int bits, long long most, int* out)
{
    const CacheShape s = cache_shape(B, Nq, H, Hkv, d, bits, most);
    out[0] = s.parts; out[1] = s.min_tiles; out[2] = s.slots; out[3] = cache_row_blocks(Nq, H, Hkv); out[4] = s.waves;
}
void t_rope(int tokens, int heads, int d, int sums, int* out)
{
    const RopeShape s = rope_shape(tokens, heads, d, sums);
    out[0] = s.blocks; out[1] = s.hg_shift; out[2] = s.shares; out[3] = rope_lanes(d); out[4] = s.rows;
}
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("ops")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "s.so")], check=True)
    lib = ctypes.CDLL(str(d / "s.so"))
    lib.t_cache.argtypes = [ctypes.c_int] * 6 + [ctypes.c_longlong, ctypes.c_void_p]

    def call(name, *a):
        out = (ctypes.c_int * 5)()
        getattr(lib, name)(*a, out)
        return list(out)
    return call


def test_chunks_fit_the_launch(rules):
    """However the lengths fall, the chunks of all sequences are no more than the launch has places for."""
    r = random.Random(1)
    for _ in range(2000):
        B, Nq, Hkv = r.choice([1, 2, 5, 48, 64, 65, 300]), r.choice([1, 2, 4, 33]), r.choice([1, 2, 8, 16])
        H, page = Hkv * r.choice([1, 3, 8]), 1 << r.randint(4, 8)
        width = int(2 ** r.uniform(0, 10))
        most = width * page
        parts, min_tiles, slots, wide, waves = rules("t_cache", B, Nq, H, Hkv, r.choice([64, 96, 128, 192, 256]), r.choice([4, 8]), most)
        assert parts >= 1 and min_tiles % 4 == 0 and waves in (1, 4) and slots >= B and wide == (2 if Nq * H // Hkv > 16 else 1)
        for lens in ([most] * B, [0] * B, [r.randint(0, most) for _ in range(B)], [most] + [1] * (B - 1)):
            tiles = [(n + 31) // 32 for n in lens]
            even, mean = -(-sum(tiles) // parts), sum(tiles) // max(sum(t > 0 for t in tiles), 1)
            n = (4 * mean + even) // max(4 * even, 1)
            chunk = max(((-(-mean // n) if n else even) + waves - 1) // waves * waves, min_tiles)
            used = sum(max(1, -(-t // chunk)) for t in tiles)
            assert used <= slots, (B, Nq, H, Hkv, most, lens[:5])
            if slots == B:
                assert used == B                        # no merge is launched


def test_rows_of_rotary_calls_are_all_taken(rules):
    """Every (token, head) is one block's, in the kernel's walk over units, shares and turns."""
    r = random.Random(2)
    for _ in range(300):
        tokens, heads, d, sums = int(2 ** r.uniform(0, 12)), r.randint(1, 80), r.choice([64, 96, 128, 192, 256]), r.randint(0, 1)
        blocks, shift, shares, lanes, turn = rules("t_rope", tokens, heads, d, sums)
        assert lanes * 16 >= d and blocks % shares == 0 and blocks > 0
        if sums:
            assert blocks <= 512 + shares
        slots, units, hg = 64 // lanes, 4 * (blocks // shares), 1 << shift
        assert hg <= slots and 1 <= turn <= (2 if sums else 4)
        if tokens * heads > 4000:
            continue
        seen = set()
        for block in range(blocks):
            share = block % shares
            for wave in range(4):
                unit = block // shares * 4 + wave
                while unit * (slots >> shift) < tokens:
                    for slot in range(slots):
                        t = unit * (slots >> shift) + (slot >> shift)
                        h0 = (slot & (hg - 1)) + share * turn * hg
                        while h0 < heads and t < tokens:
                            for u in range(turn):
                                if h0 + u * hg < heads:
                                    assert (t, h0 + u * hg) not in seen
                                    seen.add((t, h0 + u * hg))
                            h0 += shares * turn * hg
                    unit += units
        assert len(seen) == tokens * heads
