"""CPU checks of the workspaces of the calls that attend to the cache with chunks, weigh its keys and evict rows: what they ask for, and that what their
kernels write there fits, however boundaries and lengths fall."""
import ctypes
import math
import random
import subprocess

import numpy as np
import pytest

from test_cache_budget_cpu import _batches
from test_ops_cpu import CSRC, L, _cache  # noqa: F401  (L: a fixture)

MIB = 1 << 20

SHIM = r"""
#include "ops.h"
using namespace attn;
extern "C" {
void t_chunk(int B, int T, int H, int Hkv, int d, long long most, long long* out)
{
    const ChunkShape s = chunk_shape(B, T, H, Hkv, d, most);
    out[0] = chunk_places(s.places, Hkv); out[1] = s.units; out[2] = s.part_tiles; out[3] = chunk_tile_keys(d); out[4] = s.few; out[5] = kChunkFewCost;
    out[6] = (long long)kChunkPartCost;
}
void t_weigh(int B, int T, int H, int Hkv, int d, long long most, long long* out)
{
    const WeighShape s = weigh_shape(B, T, T, H, Hkv, d, most);
    out[0] = s.split; out[1] = s.parts; out[2] = weigh_keys(d); out[3] = weigh_rows(d); out[4] = kWeighFew; out[5] = kWeighRound;
}
}
"""


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    d = tmp_path_factory.mktemp("scratch")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "s.so")], check=True)
    lib = ctypes.CDLL(str(d / "s.so"))

    def call(name, B, T, H, Hkv, d, most):
        out = (ctypes.c_longlong * 8)()
        getattr(lib, name)(B, T, H, Hkv, d, ctypes.c_longlong(most), out)
        return list(out)
    return call


def _more_batches(r):
    """Those of the plans' tests, and many equal sequences whose rows or keys are divided by just more than one."""
    yield from _batches(r)
    for _ in range(500):
        B, n = r.choice([1, 3, 17, 65, 200, 1000]), int(2 ** r.uniform(0, 11))
        most = int(2 ** r.uniform(8, 16))
        m = r.randint(most // 2, most)
        yield B, B * n, [n] * B, [m] * B, most


def test_weigh_parts_fit(shapes):
    """Sums go by the workspace only for sequences whose rows are divided; these are no more than there is room for."""
    r, f32 = random.Random(6), np.float32
    most_used = 0.0
    for B, T, nq, lens, most in _more_batches(r):
        Hkv, G, d = r.choice([1, 2, 8, 16]), r.choice([1, 3, 4, 8]), r.choice([64, 128, 192, 256])
        split, room, keys, rows, few_rows, round_ = shapes("t_weigh", B, T, Hkv * G, Hkv, d, most)[:6]
        many = [(-(-m // keys), -(-n * G // rows)) for n, m in zip(nq, lens) if n * G > few_rows]
        share = max(2, math.ceil(f32(sum(s * t for s, t in many)) * f32(Hkv) / f32(round_))) if split else 1 << 30
        used = sum(s * n for s, t in many for n in [(t + share // 2) // share] if n > 1) * Hkv
        assert used <= room <= 3 * round_ // 2, (B, T, Hkv, G, d, most)
        most_used = max(most_used, used / max(room, 1))
    assert most_used > 0.7


def test_weigh_sizes(L):  # noqa: F811
    """A megabyte and a half at most, whatever the batch and the table's width."""
    c = dict(Hkv=8, page=64, pages=1 << 19)
    size = lambda B, N, width, packed: L.attn_cache_weigh_workspace_bytes(ctypes.byref(_cache(**c)), B, N, 32, width, packed)
    for B in (1, 32, 256, 1024, 8192):
        for width in (1, 512, 2048):
            assert 256 <= size(B, B, width, 1) <= 3 * MIB // 2 and size(B, 1, width, 0) == 256
    assert size(1, 2048, 512, 1) <= 3 * MIB // 2


def test_chunk_parts_fit(shapes):
    """Only sequences with more than one part write results of parts; these are no more than there is room for.  Boundaries may be nonsense too: sequences
    that share queries have more rows than T, of which the first units have blocks."""
    r, f32 = random.Random(7), np.float32
    most_used = 0.0
    for B, T, nq, lens, most in _more_batches(r):
        shared = r.random() < 0.2
        if shared:
            T = max(1, max(nq))
        Hkv, G, d = r.choice([1, 2, 8, 16, 600]), r.choice([1, 3, 4, 8]), r.choice([64, 128, 192, 256])
        mine, units, room, keys, few_rows, few_cost, part_cost = shapes("t_chunk", B, T, Hkv * G, Hkv, d, most)[:7]
        if not mine:
            assert room == 0
            continue
        seqs = []                                              # row tiles, steps, cost of a step, tiles of 32 rows in a unit
        for n, m in zip(nq, lens):
            few = n * G <= few_rows
            seqs.append((-(-n * G // (32 if few else 128)), -(-m // (128 if few else keys)), few_cost if few else 4, 1 if few else 4))
        per_unit = f32(part_cost) / f32(max(sum(s[0] for s in seqs if s[2] == 4) * Hkv, 1))

        def parts(s, per):
            n = math.ceil(float(f32(s[1]) * f32(min(f32(s[2]) * per, f32(0.25))) - f32(0.01)))
            return max(1, n if s[2] != 4 else min(n, int(math.sqrt(f32(s[1]) * per_unit))))
        per = f32(mine) / max(f32(sum(f32(s[0]) * f32(s[1]) * f32(s[2]) for s in seqs)), f32(1))
        for _ in range(3):
            if sum(s[0] * parts(s, per) for s in seqs) <= mine:
                break
            per = f32(per * f32(0.8))
        unit = used = 0
        for s in seqs:
            n = parts(s, per)
            if n > 1:
                used += max(0, min(s[0] * n, units - unit)) * s[3]
            unit += s[0] * n
        assert used <= room, (B, T, Hkv, G, d, most, shared)
        if not shared and unit <= units:
            most_used = max(most_used, used / room)
    assert most_used > 0.4


def test_chunk_sizes(L):  # noqa: F811
    """Of many single tokens: two parts of 128 rows for every place of a round, and where a sequence's parts are."""
    c = dict(Hkv=8, page=64, pages=1 << 19)
    size = lambda B, T, width: L.attn_cache_chunk_workspace_bytes(ctypes.byref(_cache(**c)), B, T, 32, width)
    assert 256 < size(32, 32, 64) <= 16 * MIB
    for B in (64, 256, 400, 512, 1024, 1900):
        for width in (64, 512):
            assert size(B, B, width) <= 66 * 2 * 8 * 128 * (128 + 2) * 4 + 16 * B + 1024
    assert size(1, 2048, 512) <= 70 * MIB and size(1, 1 << 14, 512) == 256


def test_evict_sizes(L):  # noqa: F811
    """Tables of up to 32 768 rows, whose lists are in LDS, ask for 64 KiB at most; wider ones for every row."""
    size = lambda B, width, **c: L.attn_cache_evict_workspace_bytes(ctypes.byref(_cache(**{**dict(Hkv=8, page=64, pages=1 << 19), **c})), B, width)
    for B in (1, 64, 1024, 65536):
        for width in (1, 64, 512):
            assert size(B, width) == min(B * 8 * width * 64 * 4, 65536)
        assert size(B, 513) == B * 8 * 513 * 64 * 4
