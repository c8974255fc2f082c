"""The rotary and cache calls in the runs that they are made for, on other streams and in captured graphs."""
import math

import numpy as np
import pytest
import torch

import ops_reference as ref

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def test_training_step(oracle):
    """A fused projection's q and k: norms and positions, attention, and back to the gradients of projection and weights.

    The chain against 64 bits from the same projection, each stage's results rounded to bf16 as the calls hand them on.  The attention's
    gradients are within 1e-2 in the 2-norm (the rule of parity.py); the norms' and rotation's backward is linear, shrinks no random
    gradient by more than the weights' spread (1.5 here), and rounds once (2^-8 at most): 2e-2."""
    import paper_2603_05451_amd as A
    B, N, H, Hkv, d = 2, 200, 4, 2, 64
    gen = torch.Generator("cpu").manual_seed(1)
    qkv, do = torch.randn(B, N, H + 2 * Hkv, d, generator=gen).to(BF), torch.randn(B, N, H, d, generator=gen).to(BF)
    w = [(1 + 0.1 * torch.randn(d, generator=gen)).to(BF) for _ in range(2)]
    x, f = qkv.cuda(), A.attn_rope_freqs(32)
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    kw = dict(offset=32, eps=1e-6, q_weight=w[0].cuda(), k_weight=w[1].cuda())
    scale = 2.0 / d ** 0.5
    qr, kr = A.attn_rope_fwd(q, k, f, **kw)
    o, lse = A.attn_fwd_strided(qr, kr, v, scale, True)
    dx = torch.empty_like(x)
    dq, dk, _ = A.attn_bwd_strided(qr, kr, v, o, do.cuda(), lse, scale, True, dv=dx[:, :, H + Hkv:])
    g = A.attn_rope_bwd(dq, dk, f, q=q, k=k, dq_in=dx[:, :, :H], dk_in=dx[:, :, H:H + Hkv], **kw)
    pos = torch.arange(N).expand(B, N)
    parts = [qkv[:, :, :H], qkv[:, :, H:H + Hkv]]
    r = [ref.rope(t, pos, f.cpu(), 32, False, 1.0, 1e-6, ww)[0].float().to(BF).double().numpy() for t, ww in zip(parts, w)]
    grads = oracle.attn_bwd(r[0], r[1], qkv[:, :, H + Hkv:].double().numpy(), do.double().numpy(), scale, True)
    want = [ref.rope_bwd(torch.from_numpy(np.ascontiguousarray(t)), y, pos, f.cpu(), 32, False, 1.0, 1e-6, ww) for t, y, ww in zip(grads, parts, w)]
    near = lambda got, t: float((got.double().cpu() - t).norm() / t.norm())
    assert near(dx[:, :, :H], want[0][0]) < 2e-2 and near(dx[:, :, H:H + Hkv], want[1][0]) < 2e-2
    assert near(g[2], want[0][1]) < 2e-2 and near(g[3], want[1][1]) < 2e-2
    assert near(dx[:, :, H + Hkv:], torch.from_numpy(grads[2])) < 1e-2


@pytest.mark.parametrize("bits,dtype", [(4, BF), (8, HF)])
def test_prompt_then_tokens(bits, dtype):
    """Requests of a serving loop: their prompts are written and read back for their own attention, then tokens follow one by one (an
    empty slot among them) and a draft of three; every result against 64 bits on the values that the cache holds by definition."""
    import paper_2603_05451_amd as A
    H, Hkv, d, page, scale = 8, 2, 128, 16, 128 ** -0.5
    gen = torch.Generator("cpu").manual_seed(bits)
    prompts, B = [37, 0, 5, 70], 4
    cache = A.attn_cache_new(40, page, Hkv, d, d, bits)
    table = torch.randperm(40, generator=gen).int().view(B, 10)
    slot = lambda b, j: int(table[b, j // page]) * page + j % page
    f = A.attn_rope_freqs(d, factor=4.0, original=64)
    held = [[torch.empty(0, Hkv, d, dtype=torch.float64) for _ in range(2)] for _ in range(B)]

    def new(shape, positions):
        q, k, v = (torch.randn(*shape, h, d, generator=gen).to(dtype) for h in (H, Hkv, Hkv))
        qr, kr = A.attn_rope_fwd(q.cuda(), k.cuda(), f, positions.cuda())
        return qr, kr, v.cuda()

    def keep(b, k, v):
        for i, x in enumerate((k, v)):
            held[b][i] = torch.cat((held[b][i], ref.values(*ref.quantise(x.cpu(), bits), bits)))

    def near(o, lse, q, b, Nq):
        n = held[b][0].shape[0]
        wo, wl, size, terms = ref.attend(q.double().cpu(), *held[b], scale, [n - Nq + i for i in range(Nq)])
        steps = ((d + 8) * terms + n / 32 + 64) * 2.0 ** -24                           # (as in test_gpu_cache.py)
        half = ref.HALF[dtype]
        assert ((lse.double().cpu() - wl).abs() <= steps + 2.0 ** -23 * wl.abs()).all()
        assert ((o.double().cpu() - wo).abs() <= half * wo.abs() + ref.TINY[dtype] + (half + 2 * steps.T[..., None]) * (size + wo.abs())).all()

    # prompts: one packed call each
    cu = torch.tensor([0, *np.cumsum(prompts)], dtype=torch.int32)
    T = int(cu[-1])
    pos = torch.cat([torch.arange(n) for n in prompts]).int()
    q, k, v = new((T,), pos)
    slots = torch.tensor([slot(b, j) for b in range(B) for j in range(prompts[b])], dtype=torch.int32)
    A.attn_cache_write(k, v, slots.cuda(), cache)
    kr, vr = A.attn_cache_read(slots.cuda(), cache, dtype)
    o, lse = A.attn_varlen_fwd(q, kr, vr, cu.cuda(), scale, True)
    for b in range(B):
        s = slice(int(cu[b]), int(cu[b + 1]))
        keep(b, k[s], v[s])
        assert torch.equal(kr[s].double().cpu(), held[b][0]) and torch.equal(vr[s].double().cpu(), held[b][1])
        if prompts[b]:
            wo = ref.attend(q[s].double().cpu(), *held[b], scale, range(prompts[b]))[0]
            assert (o[s].double().cpu() - wo).norm() < 1e-2 * wo.norm()
    # tokens: request 1 never has any
    for step, Nq in enumerate([1, 1, 1, 3, 1]):
        lens = [0 if b == 1 else held[b][0].shape[0] for b in range(B)]
        pos = torch.tensor([[n + i for i in range(Nq)] for n in lens], dtype=torch.int32)
        q, k, v = new((B, Nq), pos)
        slots = torch.tensor([[-1 if b == 1 else slot(b, lens[b] + i) for i in range(Nq)] for b in range(B)], dtype=torch.int32)
        A.attn_cache_write(k.reshape(-1, Hkv, d), v.reshape(-1, Hkv, d), slots.view(-1).cuda(), cache)
        now = torch.tensor([0 if b == 1 else lens[b] + Nq for b in range(B)], dtype=torch.int32)
        o, lse = A.attn_cache_fwd(q, cache, table.cuda(), now.cuda(), scale, True)
        for b in range(B):
            if b == 1:
                assert (o[b] == 0).all() and torch.isneginf(lse[b]).all()
                continue
            keep(b, k[b], v[b])
            near(o[b], lse[b], q[b], b, Nq)


def _step(A, s):
    """One decode step into given buffers."""
    A.attn_rope_fwd(s["q"], s["k"], s["f"], s["pos"], eps=1e-6, q_weight=s["w"], k_weight=s["w"], q_out=s["qr"], k_out=s["kr"])
    A.attn_cache_write(s["kr"].view(-1, *s["kr"].shape[2:]), s["v"].view(-1, *s["v"].shape[2:]), s["slots"], s["cache"])
    A.attn_cache_fwd(s["qr"], s["cache"], s["table"], s["lens"], 0.1, True, o=s["o"], lse=s["lse"], workspace=s["ws"])
    A.attn_cache_read(s["slots"], s["cache"], BF, k=s["kb"], v=s["vb"])
    s["g"] = A.attn_rope_bwd(s["qr"], s["kr"], s["f"], s["pos"], eps=1e-6, q=s["q"], k=s["k"], q_weight=s["w"], k_weight=s["w"],
                             dq_in=s["dq"], dk_in=s["dk"], workspace=s["wr"])


def _buffers(A, B=5, H=8, Hkv=2, d=128, page=32, width=60):
    e = lambda *shape, dtype=BF: torch.zeros(*shape, dtype=dtype, device="cuda")
    s = dict(q=e(B, 1, H, d), k=e(B, 1, Hkv, d), v=e(B, 1, Hkv, d), qr=e(B, 1, H, d), kr=e(B, 1, Hkv, d), o=e(B, 1, H, d), dq=e(B, 1, H, d), dk=e(B, 1, Hkv, d),
             kb=e(B, Hkv, d), vb=e(B, Hkv, d), lse=e(B, H, 1, dtype=torch.float32), w=1 + 0 * e(d), f=A.attn_rope_freqs(d), pos=e(B, 1, dtype=torch.int32),
             slots=e(B, dtype=torch.int32), lens=e(B, dtype=torch.int32), table=torch.randperm(B * width, generator=torch.Generator().manual_seed(1)).int().view(B, width).cuda(),
             cache=A.attn_cache_new(B * width, page, Hkv, d, d, 4), wr=e(A.attn_rope_workspace_bytes(B, 1, H, Hkv, d), dtype=torch.uint8))
    s["ws"] = e(A.attn_cache_workspace_bytes(s["cache"], B, 1, H, width), dtype=torch.uint8)
    g = torch.Generator("cpu").manual_seed(2)
    for t in (s["cache"].k, s["cache"].v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g).to(torch.uint8))
    for t in (s["cache"].k_scale, s["cache"].v_scale):
        t.copy_(torch.randint(124, 128, t.shape, generator=g).to(torch.uint8))
    return s


def _fill(s, seed, lens):
    g = torch.Generator("cpu").manual_seed(seed)
    for n in ("q", "k", "v"):
        s[n].copy_(torch.randn(s[n].shape, generator=g).to(BF))
    page, table = 32, s["table"].cpu()
    s["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
    s["pos"].copy_(torch.tensor([[n] for n in lens], dtype=torch.int32))
    s["slots"].copy_(torch.tensor([-1 if n == 0 else int(table[b, (n - 1) // page]) * page + (n - 1) % page for b, n in enumerate(lens)], dtype=torch.int32))


OUT = ("qr", "kr", "o", "lse", "kb", "vb", "dq", "dk")


def test_captured_and_replayed():
    """A decode step in a graph, replayed on other inputs, lengths and pages, with eager work and synchronizations between: the eager results, bit for
    bit; another graph that uses the same workspaces beside it."""
    import paper_2603_05451_amd as A
    s, e = _buffers(A), _buffers(A)
    lens = ([1, 0, 300, 1900, 33], [1500, 1500, 1500, 1500, 1500], [0, 0, 0, 0, 1], [64, 65, 1920, 31, 1024])
    _fill(s, 0, lens[0])
    _step(A, s)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            _step(A, s)
        torch.cuda.current_stream().wait_stream(side)
        graphs.append((g, s["g"]))
    for i, n in enumerate(lens * 2):
        for x in (s, e):
            _fill(x, 10 + i, n)
            x["cache"].k.copy_(s["cache"].k), x["cache"].k_scale.copy_(s["cache"].k_scale), x["cache"].v.copy_(s["cache"].v), x["cache"].v_scale.copy_(s["cache"].v_scale)
        s["ws"].fill_(255)                                  # contents are ignored
        s["wr"].fill_(255)
        _step(A, e)
        torch.cuda.synchronize()
        g, weights = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        for name in OUT:
            assert torch.equal(torch.nan_to_num(s[name].float()), torch.nan_to_num(e[name].float())), (i, name)
        assert all(torch.equal(a, b) for a, b in zip(s["cache"], e["cache"]))
        assert torch.equal(weights[2], e["g"][2]) and torch.equal(weights[3], e["g"][3])


def test_two_streams_at_once():
    """The same step of two requests' buffers on two streams, many times over: each has its own results."""
    import paper_2603_05451_amd as A
    s = [_buffers(A), _buffers(A)]
    want = []
    for i, x in enumerate(s):
        _fill(x, 20 + i, [700, 1200, 5, 0, 1900] if i else [1, 2, 3, 1800, 64])
        _step(A, x)
        torch.cuda.synchronize()
        want.append([x[n].clone() for n in OUT])
        for n in OUT:
            x[n].fill_(7)
    streams = [torch.cuda.Stream() for _ in s]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, st in zip(s, streams):
            with torch.cuda.stream(st):
                _step(A, x)
    torch.cuda.synchronize()
    for x, w in zip(s, want):
        for n, t in zip(OUT, w):
            assert torch.equal(x[n], t), n
