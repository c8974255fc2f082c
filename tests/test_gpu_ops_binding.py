"""GPU tests of the native marshalling of the rotary and cache calls against the Python text of the same functions."""
import pytest
import torch

from test_gpu_binding import _both, _t

pytestmark = pytest.mark.gpu


def _cache(A, bits):
    c = A.attn_cache_new(6, 16, 2, 64, 64, bits)
    g = torch.Generator("cpu").manual_seed(bits)
    for t, hi in zip(c, (0x47, 128, 0x47, 128)):
        t.copy_(torch.randint(120 if hi == 128 else 0, hi, t.shape, generator=g).to(torch.uint8))
    return c


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_same_outputs(monkeypatch, dtype):
    q, k = _t(2, 9, 4, 64, dtype=dtype), _t(2, 9, 2, 64, dtype=dtype, seed=1)
    w, f = _t(64, dtype=dtype), torch.rand(16).cuda()
    pos = torch.arange(18, dtype=torch.int32, device="cuda").view(2, 9)
    slots = torch.arange(18, dtype=torch.int32, device="cuda")
    table, lens = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3), torch.tensor([40, 7], dtype=torch.int32, device="cuda")
    flat = lambda t: t.reshape(18, *t.shape[2:])

    def calls(A):
        out = list(A.attn_rope_fwd(q, k, f, pos, True, 8, 1.5, 1e-6, w, w))
        out += [A.attn_rope_fwd(q[:, :, 1:3], None, f)[0], *A.attn_rope_fwd(flat(q), flat(k), f, pos.view(-1), eps=0.25, k_weight=w)]
        o = torch.empty(2, 4, 9, 64, dtype=dtype, device="cuda").transpose(1, 2)
        r = A.attn_rope_fwd(q, k, f, pos[0], q_out=o)
        assert r[0] is o
        out += r
        out += [t for t in A.attn_rope_bwd(q, k, f, pos, eps=1e-6, q=q, k=k, q_weight=w) if t is not None]
        out += [t for t in A.attn_rope_bwd(q, None, f, pos) if t is not None]
        for bits in (4, 8):
            c = _cache(A, bits)
            assert A.attn_cache_write(flat(k), flat(q)[:, 1:3], slots, c) is None
            out += [*c, *A.attn_cache_read(slots, c, dtype)]
            out += A.attn_cache_fwd(q[:, :1], c, table, lens, 0.125, True)
            lse, ws = torch.empty(2, 4, 9, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
            r = A.attn_cache_fwd(q, c, table, lens, 0.125, False, o=o.clone(), lse=lse, workspace=ws)
            assert r[1] is lse
            out += r
        return out

    native, python, results = _both(monkeypatch, calls)
    assert [n for n, r in results] == ["rope_fwd"] * 4 + ["rope_bwd"] * 2 + ["cache_write", "cache_read", "cache_fwd", "cache_fwd"] * 2
    assert all(r is not None and (r == 0 or type(r) is tuple) for n, r in results)
    assert len(native) == len(python) == 2 + 1 + 2 + 2 + 3 + 1 + 2 * (4 + 2 + 2 + 2)
    for i, (x, y) in enumerate(zip(native, python)):
        assert type(x) is torch.Tensor and x.shape == y.shape and x.stride() == y.stride() and x.dtype == y.dtype, i
        assert torch.equal(x, y) and not x.requires_grad, i
    assert all(torch.isfinite(x.float()).all() for x in native)


def test_same_refusals(monkeypatch):
    import paper_2603_05451_amd as A
    q, k, w, f = _t(2, 9, 4, 64), _t(2, 9, 2, 64), _t(64), torch.rand(16).cuda()
    slots, table, lens = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((9,), (2, 3), (2,)))
    c = A.attn_cache_new(6, 16, 2, 64, 64)
    bad = [lambda A: A.attn_rope_fwd(q, k.half(), f), lambda A: A.attn_rope_fwd(q, k[:1], f), lambda A: A.attn_rope_fwd(q, k, f.half()), lambda A: A.attn_rope_fwd(q, k, f[None]),
           lambda A: A.attn_rope_fwd(q, k, f, slots[:8]), lambda A: A.attn_rope_fwd(q, k, f, q_weight=w), lambda A: A.attn_rope_fwd(q, None, f, eps=1.0, k_weight=w),
           lambda A: A.attn_rope_fwd(q, k, f, offset=40), lambda A: A.attn_rope_fwd(q, k, f, offset=4), lambda A: A.attn_rope_fwd(q, k, f, eps=-1.0), lambda A: A.attn_rope_fwd(q, k, f, offset=-8),
           lambda A: A.attn_rope_fwd(q, k, f, q_out=k), lambda A: A.attn_rope_fwd(q, None, f, k_out=k), lambda A: A.attn_rope_fwd(q, k, f, amplitude=float("nan")),
           lambda A: A.attn_rope_bwd(q, k, f, eps=1.0), lambda A: A.attn_rope_bwd(q, k, f, eps=1.0, q=q, k=q), lambda A: A.attn_rope_bwd(q, k, f[:3]),
           lambda A: A.attn_cache_write(k[0], k[0], slots[:8], c), lambda A: A.attn_cache_write(k[0], q[0], slots, c), lambda A: A.attn_cache_write(k[0], k[0], slots.long(), c),
           lambda A: A.attn_cache_read(slots[None], c, torch.bfloat16), lambda A: A.attn_cache_read(slots, c._replace(k=c.v_scale), torch.float16), lambda A: A.attn_cache_read(slots[:0], c, torch.float16),
           lambda A: A.attn_cache_fwd(q, c, table, lens, -1.0, True), lambda A: A.attn_cache_fwd(q[:, :, :3], c, table, lens, 0.1, True), lambda A: A.attn_cache_fwd(q, c, table[:1], lens, 0.1, True),
           lambda A: A.attn_cache_fwd(q, c, table, lens.cpu(), 0.1, True), lambda A: A.attn_cache_fwd(q, c, table, lens, 0.1, True, workspace=w)]
    for i, call in enumerate(bad):
        def said(A):
            with pytest.raises((ValueError, A.AttnError)) as e:
                call(A)
            return type(e.value), str(e.value)
        native, python, results = _both(monkeypatch, said)
        assert native == python, i
        assert all(r is None or (type(r) is int and r < 0 and native[0].__name__ == "AttnError") for n, r in results), i


def test_left_to_the_python_text(monkeypatch):
    """A stream of the caller's, numbers that are no floats, outputs of the backward pass: the results of the plain call."""
    import paper_2603_05451_amd as A
    q, f = _t(2, 9, 4, 64), torch.rand(16).cuda()
    want, back = A.attn_rope_fwd(q, None, f)[0], A.attn_rope_bwd(q, None, f)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = A.attn_rope_fwd(q, None, f, stream=side)[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(A.attn_rope_fwd(q, None, f, amplitude=1)[0], want)
    mine = torch.empty_like(q)
    assert A.attn_rope_bwd(q, None, f, dq_in=mine)[0] is mine and torch.equal(mine, back)
