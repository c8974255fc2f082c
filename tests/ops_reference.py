"""Definitions in 64 bits of the rotary, cache and cache-attention calls, for the tests: numpy and torch float64 on the CPU."""
import math

import torch

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
E4M3 = torch.tensor([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)], dtype=torch.float64)
E4M3[127] = math.nan
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step, relative
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}             # half of fp16's smallest step


def pairs(rot, offset, inter):
    i = torch.arange(rot // 2)
    return (offset + 2 * i, offset + 2 * i + 1) if inter else (offset + i, offset + rot // 2 + i)


def turn(x, positions, freqs, offset, inter, amplitude, back=False):
    """x [..., N, heads, d] float64, positions [..., N]."""
    a = positions.double()[..., None, None] * freqs.double()
    c, s = torch.cos(a) * amplitude, torch.sin(a) * amplitude * (-1 if back else 1)
    i, j = pairs(2 * freqs.numel(), offset, inter)
    y = x.clone()
    y[..., i], y[..., j] = c * x[..., i] - s * x[..., j], s * x[..., i] + c * x[..., j]
    return y


def rope(x, positions, freqs, offset, inter, amplitude, eps, w):
    """-> (y, what an element's error is relative to: the sizes of what it is the sum of)."""
    x = x.double()
    if eps is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        x = x if w is None else x * w.double()
    y = turn(x, positions, freqs, offset, inter, amplitude)
    return y, spread(x.abs(), freqs, offset, inter, amplitude)


def spread(x, freqs, offset, inter, amplitude):
    i, j = pairs(2 * freqs.numel(), offset, inter)
    y = x.clone()
    y[..., i] = y[..., j] = (x[..., i] + x[..., j]) * abs(amplitude)
    return y


def rope_bwd(dy, x, positions, freqs, offset, inter, amplitude, eps, w):
    """-> (dx, dw or None, sizes as above of dx and of dw)."""
    g = turn(dy.double(), positions, freqs, offset, inter, amplitude, back=True)
    size = spread(dy.double().abs(), freqs, offset, inter, amplitude)
    if eps is None:
        return g, None, size, None
    x = x.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    over = tuple(range(x.dim() - 1))
    dw, dw_size = (g * x * r).sum(over), (size * x.abs() * r).sum(over)
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double()
    gw, sw = g * w, size * w.abs()
    dx = r * (gw - x * r * r * (gw * x).mean(-1, keepdim=True))
    return dx, dw, r * (sw + x.abs() * r * r * (sw * x.abs()).mean(-1, keepdim=True)), dw_size


def quantise(x, bits):
    """x [..., d] -> (codes [..., d], scale bytes [..., d / 32]) as integers, by search."""
    grid, top = (E2M1, 7.0) if bits == 4 else (E4M3[:127], 464.0)
    b = x.double().unflatten(-1, (-1, 32))
    amax = torch.nan_to_num(b.abs(), nan=math.inf, posinf=math.inf).amax(-1, keepdim=True)
    bad = torch.isinf(amax)
    e = torch.full_like(amax, -127.0)
    for k in range(-126, 128):                  # the least power that fits
        e = torch.where((amax < top * 2.0 ** (k - 1)) if bits == 4 else (amax <= top * 2.0 ** (k - 1)), e, float(k))
    a = torch.where(bad, 0.0, b.abs() / 2.0 ** e)
    far = (a[..., None] - grid).abs()
    near = far.amin(-1, keepdim=True)
    even = torch.arange(len(grid)) % 2 == 0
    code = torch.where((far == near) & even, 0, torch.where(far == near, 1, 2)).argmin(-1)
    code = code + torch.where(torch.signbit(b) & ~bad, 8 if bits == 4 else 128, 0)
    return code.flatten(-2), torch.where(bad, 255, e.long() + 127).squeeze(-1)


def values(code, scale, bits):
    grid = E2M1 if bits == 4 else E4M3
    v = torch.cat((grid, -grid))[code.long()].unflatten(-1, (-1, 32)) * (2.0 ** (scale.double() - 127))[..., None]
    return torch.where((scale == 255)[..., None], math.nan, v).flatten(-2)


def unpack(raw, bits):
    return raw.long() if bits == 8 else torch.stack((raw.long() & 15, raw.long() >> 4), -1).flatten(-2)


def pack(code, bits):
    code = code.to(torch.uint8)
    return code if bits == 8 else code[..., 0::2] | code[..., 1::2] << 4


def rows(codes, scales, slots, bits):
    """Rows [len(slots), Hkv, d] of a cache (CPU tensors)."""
    page = codes.shape[2]
    at = slots.long()
    return values(unpack(codes[at // page, :, at % page], bits), scales[at // page, :, at % page], bits)


def attend(q, k, v, scale, limits):
    """q [Nq, H, d], k [n, Hkv, d], v [n, Hkv, dv] float64, query i sees keys j <= limits[i] -> (o, lse [H, Nq], size of what o is the
    sum of, size of the scores' terms [H, Nq])."""
    Nq, H, _ = q.shape
    G = H // k.shape[1] if k.numel() else 1
    o = torch.zeros(Nq, H, v.shape[-1], dtype=torch.float64)
    lse = torch.full((H, Nq), -math.inf, dtype=torch.float64)
    size, terms = o.clone(), torch.zeros(H, Nq, dtype=torch.float64)
    for i in range(Nq):
        n = int(limits[i]) + 1
        if n <= 0:
            continue
        for h in range(H):
            kk, vv = k[:n, h // G], v[:n, h // G]
            s = kk @ q[i, h] * scale
            lse[h, i] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[h, i])
            o[i, h], size[i, h] = p @ vv, p @ vv.abs()
            terms[h, i] = (kk.abs() @ q[i, h].abs() * scale).max()
    return o, lse, size, terms
