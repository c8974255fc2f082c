"""GPU tests of attn_rope_fwd and attn_rope_bwd against their definitions in 64 bits.

Tolerance of an element: half a step of its type for the one rounding at the end, and the fp32 arithmetic in front: cos and sin are
off by at most 2^-22 (the reduced angle's rounding to fp32, 2^-23.3 radians, and the functions'), a sum over the head's d dims by at
most d 2^-24 of the sum of its terms' sizes (half of that behind the square root), some ten products by 2^-24 each; together below
(d + 64) 2^-24 of the sizes of what the element is a sum of, which the definitions return beside it.  An angle itself (in turns, in
64 bits, with a rounded 1 / 2 pi) is off by at most 2^-51 of its size, as is the definition's."""
import pytest
import torch

import ops_reference as ref

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def _gen(seed):
    return torch.Generator("cpu").manual_seed(seed)


def _view(gen, B, N, heads, d, dtype, layout, wide=1):
    """[B, N, heads, d] on the CPU and as a GPU view of that layout."""
    x = torch.randn(B, N, heads, d, generator=gen).to(dtype)
    if layout == "bhnd":
        return x, x.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "slice":                                   # of a wider buffer: heads and dims padded
        buf = torch.full((B, N + 1, heads + 2, d + 8), 7.0, dtype=dtype, device="cuda")
        buf[:, :N, 1:1 + heads, :d] = x.cuda()
        return x, buf[:, :N, 1:1 + heads, :d]
    return x, x.cuda()


def _close(got, want, size, dtype, d, angle=0.0):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    bound = ref.HALF[dtype] * want.abs() + ref.TINY[dtype] + ((d + 64) * 2.0 ** -24 + 2.0 ** -50 * angle) * size
    worst = ((got - want).abs() - bound).max()
    assert worst <= 0, worst


CASES = [
    # B, N, H, Hkv, d, rot, offset, inter, norm ("" none, "w" weights, "1" ones), dtype, layout, positions, amplitude
    (1, 1, 1, 1, 64, 64, 0, False, "", BF, "dense", None, 1.0),
    (1, 1, 32, 8, 128, 128, 0, False, "w", BF, "dense", "batch", 1.0),
    (2, 37, 5, 1, 128, 128, 0, False, "w", BF, "bhnd", "batch", 1.3),
    (2, 37, 5, 1, 128, 128, 0, True, "w", HF, "slice", "shared", 1.0),
    (3, 19, 3, 3, 64, 32, 0, True, "w", HF, "slice", "batch", 0.5),
    (3, 19, 3, 3, 64, 16, 40, False, "1", BF, "dense", None, 1.0),
    (1, 130, 7, 2, 96, 96, 0, False, "w", BF, "slice", "batch", 1.0),
    (1, 130, 7, 2, 96, 80, 8, True, "", HF, "bhnd", "shared", 1.0),
    (2, 66, 16, 16, 192, 64, 128, False, "", BF, "dense", "batch", 1.0),
    (2, 66, 4, 2, 192, 176, 16, True, "w", BF, "slice", "batch", -2.0),
    (1, 257, 9, 3, 256, 256, 0, False, "w", HF, "dense", "batch", 1.0),
    (1, 257, 2, 1, 256, 48, 120, True, "1", BF, "bhnd", "batch", 1.0),
    (5, 700, 2, 1, 64, 64, 0, False, "w", BF, "dense", None, 1.0),
    (1, 4100, 8, 4, 128, 64, 64, False, "w", BF, "slice", "batch", 1.0),
]


def _make(case, seed=0):
    B, N, H, Hkv, d, rot, offset, inter, norm, dtype, layout, pos, amp = case
    gen = _gen(seed)
    q, qg = _view(gen, B, N, H, d, dtype, layout)
    k, kg = _view(gen, B, N, Hkv, d, dtype, layout)
    f = (10000.0 ** (-torch.arange(0, rot, 2).double() / rot)).float()
    if pos is None:
        positions, full = None, torch.arange(N).expand(B, N)
    else:
        positions = torch.randint(-50, 200000, (B, N) if pos == "batch" else (N,), generator=gen).int()
        full = positions.expand(B, N)
    w = [(1 + 0.3 * torch.randn(d, generator=gen)).to(dtype) if norm == "w" else None for _ in range(2)]
    eps = 1e-5 if norm else None
    kw = dict(positions=None if positions is None else positions.cuda(), interleaved=inter, offset=offset, amplitude=amp, eps=eps,
              q_weight=None if w[0] is None else w[0].cuda(), k_weight=None if w[1] is None else w[1].cuda())
    return (q, qg), (k, kg), f, full, (offset, inter, amp, eps), w, kw, gen


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    import paper_2603_05451_amd as A
    (q, qg), (k, kg), f, full, args, w, kw, _ = _make(case)
    qo, ko = A.attn_rope_fwd(qg, kg, f.cuda(), **kw)
    assert qo.is_contiguous() and qo.shape == q.shape and ko.shape == k.shape and qo.dtype == q.dtype
    for got, x, ww in ((qo, q, w[0]), (ko, k, w[1])):
        want, size = ref.rope(x, full, f, *args, ww)
        _close(got, want, size, x.dtype, x.shape[-1], float(full.abs().max()))
    assert torch.equal(qg.cpu(), q) and torch.equal(kg.cpu(), k)


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    import paper_2603_05451_amd as A
    (q, qg), (k, kg), f, full, args, w, kw, gen = _make(case, 1)
    B, N, H, Hkv, d, layout, dtype = case[0], case[1], case[2], case[3], case[4], case[10], case[9]
    dq, dqg = _view(gen, B, N, H, d, dtype, layout)
    dk, dkg = _view(gen, B, N, Hkv, d, dtype, layout)
    saved = dict(q=qg, k=kg) if args[3] is not None else {}
    got = A.attn_rope_bwd(dqg, dkg, f.cuda(), **kw, **saved)
    for i, (dy, x, ww) in enumerate(((dq, q, w[0]), (dk, k, w[1]))):
        dx, dw, size, dw_size = ref.rope_bwd(dy, x, full, f, *args, ww)
        _close(got[i], dx, size, dtype, d, float(full.abs().max()))
        if ww is None:
            assert got[2 + i] is None
        else:
            # a lane's rows one after the other (at most rows / 8 of them), the row slots, waves, blocks (16 at a time, at most 65 turns)
            rows = B * N * (H + Hkv)
            steps = min(rows, 4100 * 12 // 8) + 64 + 4 + 65 + 16 + d
            off = (got[2 + i].double().cpu() - dw).abs()
            assert got[2 + i].dtype == torch.float32 and (off <= (steps * 2.0 ** -24 + 2.0 ** -50 * float(full.abs().max())) * dw_size).all()
    again = A.attn_rope_bwd(dqg, dkg, f.cuda(), **kw, **saved)
    assert all(a is b or torch.equal(a, b) for a, b in zip(got, again))


def test_far_positions():
    """The angle of a far position is that of its exact product with the frequency."""
    import paper_2603_05451_amd as A
    q = torch.randn(1, 6, 2, 64, generator=_gen(3)).to(BF)
    pos = torch.tensor([0, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31), -12345679], dtype=torch.int32)
    f = (500000.0 ** (-torch.arange(0, 64, 2).double() / 64)).float()
    got, none = A.attn_rope_fwd(q.cuda(), None, f.cuda(), pos.cuda())
    assert none is None
    want, size = ref.rope(q, pos[None], f, 0, False, 1.0, None, None)
    _close(got, want, size, BF, 64, 2.0 ** 31)


def test_in_place_packed_and_one_tensor():
    import paper_2603_05451_amd as A
    gen = _gen(4)
    f = A.attn_rope_freqs(64)
    q, k = torch.randn(300, 6, 128, generator=gen).to(HF).cuda(), torch.randn(300, 2, 128, generator=gen).to(HF).cuda()
    w = torch.rand(128, generator=gen).to(HF).cuda()
    pos = torch.randint(0, 5000, (300,), generator=gen).int().cuda()
    kw = dict(offset=16, eps=1e-6, q_weight=w)
    want = A.attn_rope_fwd(q, k, f, pos, **kw)
    assert want[0].shape == (300, 6, 128)
    alone = A.attn_rope_fwd(q, None, f, pos, **kw)[0]
    assert torch.equal(alone, want[0])
    qkv = torch.cat((q, k), dim=1)
    a, b = qkv[:, :6], qkv[:, 6:]
    got = A.attn_rope_fwd(a, b, f, pos, q_out=a, k_out=b, **kw)
    assert got[0] is a and torch.equal(a, want[0]) and torch.equal(b, want[1])
    g = [torch.randn(t.shape, generator=gen).to(HF).cuda() for t in (q, k)]
    want = A.attn_rope_bwd(*g, f, pos, q=q, k=k, **kw)
    assert want[3] is None and want[2].shape == (128,)
    got = A.attn_rope_bwd(*g, f, pos, q=q, k=k, dq_in=g[0], dk_in=g[1], **kw)
    assert got[0] is g[0] and all(torch.equal(x, y) for x, y in zip(got[:3], want[:3]))


def test_offsets_beyond_32_bits():
    """Tokens further apart than 2^31 elements, and a sequence behind that; inputs, gradients and outputs."""
    import paper_2603_05451_amd as A
    gen = _gen(5)
    f, w = A.attn_rope_freqs(64), torch.rand(64, generator=gen).to(BF).cuda()
    x, dy = (torch.randn(2, 2, 3, 64, generator=gen).to(BF).cuda() for _ in range(2))
    far = torch.empty((1 << 32) + (1 << 20), dtype=BF, device="cuda").as_strided((2, 2, 3, 64), ((1 << 31) + 512, 1 << 31, 64, 1))
    want = A.attn_rope_fwd(x, None, f, eps=1e-6, q_weight=w)[0]
    back = A.attn_rope_bwd(dy, None, f, eps=1e-6, q=x, q_weight=w)
    far.copy_(x)
    assert torch.equal(A.attn_rope_fwd(far, None, f, eps=1e-6, q_weight=w)[0], want)
    assert torch.equal(A.attn_rope_bwd(dy, None, f, eps=1e-6, q=far, q_weight=w)[0], back[0])
    assert torch.equal(A.attn_rope_fwd(x, None, f, eps=1e-6, q_weight=w, q_out=far)[0], want)
    far.copy_(dy)
    got = A.attn_rope_bwd(far, None, f, eps=1e-6, q=x, q_weight=w, dq_in=far)
    assert got[0] is far and torch.equal(far, back[0]) and torch.equal(got[2], back[2])


def test_zero_rows_and_rows_that_are_no_numbers():
    """A row of zeros has a finite norm; one NaN or infinity stays in its own row."""
    import paper_2603_05451_amd as A
    q = torch.randn(1, 40, 3, 64, generator=_gen(6)).to(BF)
    q[0, 7, 1] = 0
    f, w = A.attn_rope_freqs(64), torch.ones(64, dtype=BF).cuda()
    clean = A.attn_rope_fwd(q.cuda(), None, f, eps=1e-6, q_weight=w)[0].cpu()
    assert (clean[0, 7, 1] == 0).all() and torch.isfinite(clean.float()).all()
    q[0, 9, 0, 5], q[0, 9, 2, 60] = float("nan"), float("inf")
    got = A.attn_rope_fwd(q.cuda(), None, f, eps=1e-6, q_weight=w)[0].cpu()
    same = torch.ones(1, 40, 3, dtype=torch.bool)
    same[0, 9, 0] = same[0, 9, 2] = False
    assert torch.equal(got[same], clean[same]) and torch.isnan(got[0, 9, 0].float()).all() and not torch.isfinite(got[0, 9, 2].float()).all()
    x = A.attn_rope_bwd(clean.cuda(), None, f, eps=1e-6, q=q.cuda())
    assert torch.isfinite(x[0].cpu()[same].float()).all()


def test_refusals_of_tensors():
    import paper_2603_05451_amd as A
    q, k, f = torch.zeros(2, 8, 4, 64, dtype=BF, device="cuda"), torch.zeros(2, 8, 2, 64, dtype=BF, device="cuda"), A.attn_rope_freqs(64)
    w, pos = torch.ones(64, dtype=BF, device="cuda"), torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    bad = [lambda: A.attn_rope_fwd(q.float(), k, f), lambda: A.attn_rope_fwd(q, k.half(), f), lambda: A.attn_rope_fwd(q, k[:, :7], f),
           lambda: A.attn_rope_fwd(q, k[..., ::2], f), lambda: A.attn_rope_fwd(q[0, 0], None, f), lambda: A.attn_rope_fwd(q, k, f.double()),
           lambda: A.attn_rope_fwd(q, k, f.cpu()), lambda: A.attn_rope_fwd(q, k, f, pos.long()), lambda: A.attn_rope_fwd(q, k, f, pos[:, :7]),
           lambda: A.attn_rope_fwd(q, k, f, q_weight=w), lambda: A.attn_rope_fwd(q, k, f, eps=1e-6, q_weight=w[:32]), lambda: A.attn_rope_fwd(q, k, f, eps=1e-6, q_weight=w.float()),
           lambda: A.attn_rope_fwd(q, None, f, eps=1e-6, k_weight=w), lambda: A.attn_rope_fwd(q, None, f, k_out=k), lambda: A.attn_rope_fwd(q, k, f, q_out=k),
           lambda: A.attn_rope_bwd(q, k, f, eps=1e-6), lambda: A.attn_rope_bwd(q, k, f, eps=1e-6, q=q), lambda: A.attn_rope_bwd(q, None, f, dk_in=k),
           lambda: A.attn_rope_bwd(q, k, f, eps=1e-6, q=q, k=k, q_weight=w, workspace=torch.zeros(9, device="cuda"))]
    for i, g in enumerate(bad):
        with pytest.raises(ValueError):
            g()
            assert False, i
    errors = [lambda: A.attn_rope_fwd(q, k, f, offset=8), lambda: A.attn_rope_fwd(q, k, f[:12]), lambda: A.attn_rope_fwd(q, k, f, eps=-1.0),
              lambda: A.attn_rope_fwd(q.expand(3, 2, 8, 4, 64)[:, 0], None, f), lambda: A.attn_rope_fwd(q[:0], None, f),
              lambda: A.attn_rope_bwd(q, k, f, eps=1e-6, q=q, k=k, q_weight=w, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))]
    for g in errors:
        with pytest.raises(A.AttnError):
            g()
