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
