"""GPU test of the cache at the end of the element types' ranges: numbers below the stated ones read back finite and within half a step,
the others infinite."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("bits,dtype,first", [(4, BF, 7 * 2.0 ** 125), (8, BF, 248 * 2.0 ** 120), (4, HF, 57344.0), (8, HF, 63488.0)])
def test_first_number_that_reads_back_infinite(bits, dtype, first):
    import paper_2603_05451_amd as A
    at = torch.tensor(first, dtype=torch.float64).to(dtype)
    below = (at.view(torch.int16) - 1).view(dtype)               # the next number towards zero
    assert float(at) == first
    rows = torch.zeros(4, 1, 64, dtype=dtype)
    rows[0, 0, 3], rows[1, 0, 3], rows[2, 0, 3], rows[3, 0, 3] = below, at, -at, torch.finfo(dtype).max
    rows[:, 0, 4] = first / 8                                    # (in the block with it: finite throughout)
    cache, slots = A.attn_cache_new(1, 16, 1, 64, 64, bits), torch.arange(4, dtype=torch.int32, device="cuda")
    A.attn_cache_write(rows.cuda(), rows.cuda(), slots, cache)
    for got in A.attn_cache_read(slots, cache, dtype):
        got = got.cpu().double()[:, 0]
        half = 2.0 ** -2 if bits == 4 else 2.0 ** -4             # of the code
        assert abs(float(got[0, 3]) - float(below)) <= half * float(below)
        assert got[1:, 3].tolist() == [math.inf, -math.inf, math.inf]
        assert torch.isfinite(got[:, 4]).all() and torch.isfinite(got[:, 32:]).all()
    if dtype == HF:                                              # (bf16 holds them)
        assert all(torch.isfinite(t.float()).all() for t in A.attn_cache_read(slots, cache, BF))
