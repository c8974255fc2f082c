"""CPU checks of the calls that attend to the cache with chunks, weigh its keys and evict rows: what the C ABI and the Python functions refuse, the
rules that share the work out, and the tests' own definitions."""
import ctypes
import math
import os
import random
import subprocess

import numpy as np
import pytest
import torch

import cache_reference as cref
from test_ops_cpu import BAD_CACHES, CSRC, FOREIGN_CACHES, L, ODD, P, _cache, _st  # noqa: F401  (L: a fixture)

TWO, WS = ctypes.c_void_p(0x1002), ctypes.c_void_p(0x1010)


def _refused(call, invalid, unsupported):
    import paper_2603_05451_amd as A
    for x in invalid:
        assert call(**x) == A.ATTN_EINVAL, x
    for x in unsupported:
        assert call(**x) == A.ATTN_EUNSUPPORTED, x
    for x in BAD_CACHES:
        assert call(c=_cache(**x)) == A.ATTN_EINVAL, x
    for x in FOREIGN_CACHES:
        assert call(c=_cache(**x)) == A.ATTN_EUNSUPPORTED, x


def test_chunk_refusals(L):  # noqa: F811
    s = _st(0, 1024, 128)

    def call(c=None, dtype=0, q=P, sq=s, o=P, so=s, lse=P, table=P, width=4, cu=P, lens=P, B=3, T=50, H=8, scale=0.1, ws=P, n=1 << 40):
        return L.attn_cache_chunk_fwd(dtype, ctypes.byref(c or _cache()), q, sq, o, so, lse, table, width, cu, lens, B, T, H, scale, 1, ws, n, None)
    _refused(call, [dict(q=None), dict(o=None), dict(lse=None), dict(table=None), dict(cu=None), dict(lens=None), dict(ws=None), dict(q=ODD), dict(o=ODD), dict(lse=TWO),
                    dict(cu=TWO), dict(lens=TWO), dict(table=TWO), dict(ws=WS), dict(width=0), dict(B=0), dict(T=0), dict(T=-1), dict(H=0), dict(H=7), dict(scale=0.0),
                    dict(scale=-1.0), dict(scale=math.nan), dict(scale=1e31), dict(sq=None), dict(so=_st(0, 1020, 128)), dict(sq=_st(0, 0, 128)), dict(so=_st(0, 1024, 0)),
                    dict(width=1000, n=256), dict(n=0)],
             [dict(dtype=2), dict(width=1 << 26), dict(B=65537), dict(T=1 << 26), dict(T=1 << 30)])
    assert L.attn_cache_chunk_fwd(0, None, P, s, P, s, P, P, 4, P, P, 3, 50, 8, 0.1, 1, P, 1 << 40, None) == -1
    size = lambda *a, **c: L.attn_cache_chunk_workspace_bytes(ctypes.byref(_cache(**c)), *a)
    assert size(3, 50, 8, 4) == 256 and size(3, 50, 8, 100) > 256 and size(3, 50, 7, 4) == 0 and size(3, 50, 8, 4, bits=3) == 0 and size(1, 1 << 14, 8, 1000) == 256


def test_weigh_refusals(L):  # noqa: F811
    s = _st(1024, 1024, 128)

    def call(c=None, dtype=0, q=P, sq=s, lse=P, w=P, table=P, width=4, cu=None, lens=P, B=3, Nq=2, H=8, scale=0.1, ws=P, n=1 << 40):
        return L.attn_cache_weigh(dtype, ctypes.byref(c or _cache()), q, sq, lse, w, table, width, cu, lens, B, Nq, H, scale, 1, 1, ws, n, None)
    for cu in (None, P):
        _refused(lambda **x: call(**{"cu": cu, **x}),
                 [dict(q=None), dict(lse=None), dict(w=None), dict(table=None), dict(lens=None), dict(ws=None), dict(q=ODD), dict(lse=TWO), dict(w=ODD), dict(cu=TWO),
                  dict(lens=TWO), dict(ws=WS), dict(width=0), dict(B=0), dict(Nq=0), dict(H=0), dict(H=7), dict(scale=0.0), dict(scale=math.inf), dict(sq=None),
                  dict(sq=_st(1024, 1020, 128)), dict(n=128), dict(Nq=1000, n=256)],
                 [dict(dtype=2), dict(width=1 << 26), dict(B=65537), dict(Nq=1 << 26)])
    assert call(sq=_st(0, 1024, 128)) == -1                    # sequences of their own need a batch stride
    size = lambda *a, **c: L.attn_cache_weigh_workspace_bytes(ctypes.byref(_cache(**c)), *a)
    assert size(3, 2, 8, 4, 0) == 256 and size(3, 2000, 8, 4, 1) > 256 and size(3, 2, 7, 4, 0) == 0 and size(3, 2, 8, 4, 0, bits=3) == 0


def test_evict_refusals(L):  # noqa: F811
    def call(c=None, w=P, table=P, width=4, lens=P, keep=ctypes.c_void_p(0x2000), recent=3, B=3, out=ctypes.c_void_p(0x3000), ws=P, n=1 << 40):
        return L.attn_cache_evict(ctypes.byref(c or _cache()), w, table, width, lens, keep, recent, B, out, ws, n, None)
    _refused(call, [dict(w=None), dict(table=None), dict(lens=None), dict(keep=None), dict(out=None), dict(ws=None), dict(w=ODD), dict(lens=TWO), dict(keep=TWO), dict(out=TWO),
                    dict(ws=WS), dict(width=0), dict(B=0), dict(recent=-1), dict(out=P), dict(out=ctypes.c_void_p(0x2000)), dict(out=ctypes.c_void_p(0x2008)), dict(out=ctypes.c_void_p(0x1ff8)), dict(n=256), dict(c=_cache(k_scale=0x1004)),
                    dict(c=_cache(v_scale=0x1001))],
             [dict(width=1 << 26), dict(width=1 << 22), dict(B=65537), dict(B=60000, c=_cache(Hkv=128))])
    size = lambda *a, **c: L.attn_cache_evict_workspace_bytes(ctypes.byref(_cache(**c)), *a)
    assert size(3, 4) == 3 * 2 * 4 * 32 * 4 and size(3, 0) == 0 and size(3, 4, bits=3) == 0


def test_python_refusals_without_a_gpu():
    import paper_2603_05451_amd as A
    c = A.attn_cache_new(2, 16, 2, 64, 64, device="cpu")
    w = A.attn_cache_weights(c)
    assert w.shape == (2, 2, 16) and w.dtype == torch.float32 and not w.any()
    q, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), lambda *s: torch.zeros(*s, dtype=torch.int32)
    for f in (lambda: A.attn_cache_chunk_fwd(q, c, i(1, 1), i(2), i(1), 0.1, True), lambda: A.attn_cache_weigh(q, torch.zeros(2, 4), w, c, i(1, 1), i(1), 0.1, True, cu_seqlens=i(2)),
              lambda: A.attn_cache_weigh(q[None], torch.zeros(1, 2, 4), w, c, i(1, 1), i(1), 0.1, True), lambda: A.attn_cache_evict(w, c, i(1, 1), i(1), i(1), 3)):
        with pytest.raises(ValueError):
            f()


# ---- how the work is shared out

SHIM = r"""
#include "ops.h"
using namespace attn;
extern "C" {
void t_chunk(int B, int T, int H, int Hkv, int d, long long most, long long* out)
{
    const ChunkShape s = chunk_shape(B, T, H, Hkv, d, most);
    out[0] = s.places; out[1] = s.units; out[2] = chunk_tile_keys(d); out[3] = s.few; out[4] = kChunkFewCost; out[5] = (long long)kChunkPartCost;
}
void t_weigh(int B, int T, int H, int Hkv, int d, long long most, long long* out)
{
    const WeighShape s = weigh_shape(B, T, T, H, Hkv, d, most);
    out[0] = s.split; out[1] = s.groups; out[2] = s.units; out[3] = weigh_keys(d); out[4] = weigh_rows(d); out[5] = kWeighFew; out[6] = kWeighRound;
}
}
"""


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    d = tmp_path_factory.mktemp("budget")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "s.so")], check=True)
    lib = ctypes.CDLL(str(d / "s.so"))

    def call(name, B, T, H, Hkv, d, most):
        out = (ctypes.c_longlong * 8)()
        getattr(lib, name)(B, T, H, Hkv, d, ctypes.c_longlong(most), out)
        return list(out)
    return call


def _batches(r):
    """(queries, keys) of batches of all kinds, with the room of the table's rows."""
    for _ in range(1500):
        B = r.choice([1, 2, 5, 26, 64, 65, 300])
        most = int(2 ** r.uniform(4, 16))
        q = int(2 ** r.uniform(0, 12))
        nq = r.choice([[q] * B, [1] * B, [r.randint(0, q) for _ in range(B)], [q] + [0] * (B - 1), [1] * (B - 1) + [q]])
        lens = r.choice([[most] * B, [r.randint(0, most) for _ in range(B)], [most] + [1] * (B - 1), [min(n, most) for n in nq]])
        yield B, max(1, sum(nq)), nq, lens, most


def test_chunk_units_fit_the_launch(shapes):
    """However boundaries and lengths fall, the parts of all row tiles are no more than the launch and its workspace have room for; the parts of a
    sequence hold all its keys."""
    r, f32 = random.Random(3), np.float32
    for B, T, nq, lens, most in _batches(r):
        Hkv, G, d = r.choice([1, 2, 8, 16]), r.choice([1, 3, 4, 8]), r.choice([64, 128, 192, 256])
        places, room, keys, few_rows, few_cost, part_cost = shapes("t_chunk", B, T, Hkv * G, Hkv, d, most)[:6]
        seqs = []
        for n, m in zip(nq, lens):
            few = n * G <= few_rows
            step = 128 if few else keys
            seqs.append((-(-n * G // (32 if few else 128)), -(-m // step), few_cost if few else 4))
        per_unit = f32(part_cost) / f32(max(sum(s[0] for s in seqs if s[2] == 4) * Hkv, 1))

        def parts(s, per):
            most_parts = math.ceil(float(f32(s[1]) * f32(min(f32(s[2]) * per, f32(0.25))) - f32(0.01)))
            return 1 if not places else max(1, most_parts if s[2] != 4 else min(most_parts, int(math.sqrt(f32(s[1]) * per_unit))))
        per = f32(1)
        if places:
            mine = places // Hkv + 1
            per = f32(mine) / max(f32(sum(f32(s[0]) * f32(s[1]) * f32(s[2]) for s in seqs)), f32(1))
            for _ in range(3):
                if sum(s[0] * parts(s, per) for s in seqs) <= mine:
                    break
                per = f32(per * f32(0.8))
        assert sum(s[0] * parts(s, per) for s in seqs) <= room, (B, T, Hkv, G, d, most)
        for s in seqs:
            n = parts(s, per)
            assert n * -(-s[1] // n) >= s[1]


def test_weigh_units_fit_the_launch(shapes):
    """The same of the shares of rows that keys are weighed by."""
    r, f32 = random.Random(4), np.float32
    for B, T, nq, lens, most in _batches(r):
        Hkv, G, d = r.choice([1, 2, 8, 16]), r.choice([1, 3, 4, 8]), r.choice([64, 128, 192, 256])
        split, groups, room, keys, rows, few_rows, round_ = shapes("t_weigh", B, T, Hkv * G, Hkv, d, most)[:7]
        steps = [-(-m // keys) if n else 0 for n, m in zip(nq, lens)]
        few, tiles = [n * G <= few_rows for n in nq], [-(-n * G // rows) for n in nq]
        of_few = sum(s for s, f in zip(steps, few) if f)
        of_many = sum(s * t for s, t, f in zip(steps, tiles, few) if not f)
        few_steps = max(1, math.ceil(f32(of_few) * f32(Hkv) / f32(round_)))
        share = max(2, math.ceil(f32(of_many) * f32(Hkv) / f32(round_))) if split else 1 << 30
        units = kinds = 0
        for s, t, f in zip(steps, tiles, few):
            g = -(-s // (few_steps if f else 1))
            n = 1 if f else max(1, (t + share // 2) // share)
            assert g == 0 or g * -(-s // g) >= s and n * -(-t // n) >= t
            units += g * n
            kinds += g
        assert units * Hkv <= room and kinds * Hkv <= groups, (B, T, Hkv, G, d, most)


# ---- the definitions that the GPU tests compare with

def test_weights_are_the_columns_of_p():
    g = cref.gen(1)
    q, k, v = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((7, 6, 64), (20, 2, 64), (20, 2, 64)))
    for causal in (True, False):
        o, lse, _, _ = cref.attend(q, k, v, 0.125, causal)
        w, off = cref.weigh(q, lse, k, 0.125, causal)
        assert (w.sum(0) - 7 * 3).abs().max() < 1e-12 and (off > 0).all() and (off < 1e-4).all()
        one = torch.zeros(20, 2, 20, dtype=torch.float64)
        for j in range(20):
            one[j, :, j] = 1                                   # o of one-hot values: rows of P
        p = cref.attend(q, k, one, 0.125, causal)[0]
        assert (w - p.view(7, 2, 3, 20).sum((0, 2)).T).abs().max() < 1e-12
        assert (torch.einsum("ihj,jc->ihc", p.view(7, 6, 20)[:, :3], v[:, 0]) - o[:, :3]).abs().max() < 1e-12


def test_places_keep_the_greatest():
    r = random.Random(2)
    for _ in range(300):
        n = r.randint(1, 40)
        w = [r.choice([0.0, -0.0, 1.0, math.inf, math.nan, r.random()]) for _ in range(n)]
        keep, recent = r.randint(-1, n + 3), r.randint(0, 12)
        to, of = cref.places(w, n, keep, recent)
        rows = list(range(n))
        for a, b in zip(to, of):
            rows[a] = b
        left = min(n, max(keep, 0))
        kept = rows[:left]
        last = min(recent, left)
        if left == n:
            assert not to
            continue
        assert len(set(kept)) == left and kept[left - last:] == list(range(n - last, n))
        assert all(i == j for i, j in enumerate(kept[:left - last]) if j < left - last)
        rank = lambda j: (math.inf if math.isnan(w[j]) else w[j], math.isnan(w[j]), -j)
        out = set(range(n - last)) - set(kept)
        assert not out or not kept[:left - last] or min(rank(j)[:2] for j in kept[:left - last]) >= max(rank(j)[:2] for j in out)
