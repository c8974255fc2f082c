"""GPU tests of the head norms of attn_rope_fwd and attn_rope_bwd where the squares of a row's numbers leave fp32's range (bf16 has its
exponents: 10^-19 and below, 10^19 and above), with eps = 0 and a small one, against the definitions in 64 bits.  Tolerance: that of
test_gpu_rope.py; bf16's half step is absolute below its smallest normal number, 2^-134, where a result may be flushed to zero, 2^-126."""
import pytest
import torch

import ops_reference as ref

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def _make(H, d, dtype, sizes, N=11):
    gen = torch.Generator("cpu").manual_seed(d + H)
    x = torch.randn(1, N, H, d, generator=gen)
    p = torch.tensor(sizes)[torch.randint(0, len(sizes), (1, N, H, 1), generator=gen)]
    x = (x.clamp(-3, 3) * 2.0 ** p).to(dtype)                    # (3 * 2^126 is below bf16's largest number)
    dy = torch.randn(1, N, H, d, generator=gen) * 2.0 ** (p / 4)
    w = (1 + 0.2 * torch.randn(d, generator=gen)).to(dtype)
    return x, dy.to(dtype), w


def _near(got, want, size, d):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -126 + (d + 64) * 2.0 ** -24 * size
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() - bound).max()


SIZES = [-126.0, -110.0, -80.0, -66.0, -64.0, -62.0, -50.0, -3.0, 0.0, 40.0, 52.0, 62.0, 64.0, 66.0, 100.0, 126.0]


@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-12])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("H,d", [(1, 64), (3, 96), (9, 128), (2, 192), (40, 256)])
def test_rows_of_any_size(H, d, inter, eps):
    import paper_2603_05451_amd as A
    x, dy, w = _make(H, d, BF, SIZES)
    f, pos = A.attn_rope_freqs(32, device="cpu"), torch.arange(11).view(1, 11)
    args = (16, inter, 1.0, eps)
    kw = dict(offset=16, interleaved=inter, eps=eps, q_weight=w.cuda())
    got = A.attn_rope_fwd(x.cuda(), None, f.cuda(), **kw)[0]
    _near(got, *ref.rope(x, pos, f, *args, w), d)
    dx, dw, size, dw_size = ref.rope_bwd(dy, x, pos, f, *args, w)
    keep = (dx.abs() < 2.0 ** 120).all(-1)                       # (a gradient may pass bf16's range; those of this test do not)
    assert keep.all()
    back = A.attn_rope_bwd(dy.cuda(), None, f.cuda(), q=x.cuda(), **kw)
    _near(back[0], dx, size, d)
    assert ((back[2].double().cpu() - dw).abs() <= (11 * H + 150 + d) * 2.0 ** -24 * dw_size).all()


def test_other_rows_keep_their_results():
    """Bit for bit, beside rows far from them; an infinite number and a NaN stay in their rows."""
    import paper_2603_05451_amd as A
    x, dy, w = _make(8, 128, BF, [0.0])
    f, kw = A.attn_rope_freqs(128), dict(eps=1e-6, q_weight=w.cuda())
    far = x.clone()
    far[0, 2, 1] *= 2.0 ** 70
    far[0, 3, 7], far[0, 5, 0, 9] = 2.0 ** 127, float("inf")
    far[0, 6, 4, 100] = float("nan")
    same = (far == x).all(-1)
    for a, b in ((A.attn_rope_fwd(x.cuda(), None, f, **kw)[0], A.attn_rope_fwd(far.cuda(), None, f, **kw)[0]),
                 (A.attn_rope_bwd(dy.cuda(), None, f, q=x.cuda(), **kw)[0], A.attn_rope_bwd(dy.cuda(), None, f, q=far.cuda(), **kw)[0])):
        assert torch.equal(a.cpu()[same], b.cpu()[same])
        assert torch.isfinite(b[0, 2, 1].float()).all() and torch.isfinite(b[0, 3, 7].float()).all()
        assert torch.isnan(b[0, 6, 4].float()).all() and not torch.isfinite(b[0, 5, 0].float()).all()


def test_zeros_with_a_small_eps():
    import paper_2603_05451_amd as A
    for dtype in (BF, HF):
        x = torch.zeros(1, 5, 3, 64, dtype=dtype, device="cuda")
        for eps in (1e-38, 1e-30, 1e-6):
            y = A.attn_rope_fwd(x, None, A.attn_rope_freqs(64), eps=eps)[0]
            assert (y == 0).all()
            g = A.attn_rope_bwd(torch.full_like(x, 2.0 ** -20), None, A.attn_rope_freqs(64), eps=eps, q=x, q_weight=torch.ones(64, dtype=dtype, device="cuda"))
            assert (g[2] == 0).all() and (dtype == HF or torch.isfinite(g[0].float()).all())
