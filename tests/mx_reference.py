"""Blocks of the 4- and 8-bit K/V cache, and attention, in float64 on the CPU: from the definitions, no code of the HIP path."""
import math

import torch

HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2
LOWEST = {4: -125, 8: -117}


def grid(bits):
    """Non-negative values of the codes 0, 1, ... ."""
    if bits == 4:
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    c = torch.arange(127)
    return torch.where(c < 8, c * 2.0 ** -9, (8 + c % 8) * 2.0 ** (c // 8 - 10)).double()


def quantize(v, bits):
    """v [..., hd]: the codes (sign in the top bit) and scale bytes of its blocks of 32."""
    g, b = grid(bits), v.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    top = torch.where(bad, 0.0, top)
    past = float(g[-1] + (g[-1] - g[-2]) / 2)
    e = torch.full(top.shape, LOWEST[bits])
    for x in range(LOWEST[bits], 128):
        lim = past * 2.0 ** x
        e = torch.where(top >= lim if bits == 4 else top > lim, x + 1, e)
    y = torch.where(bad[..., None], 0.0, b).abs() * 2.0 ** -e[..., None].double()
    hi = torch.searchsorted(g, y).clamp(1, len(g) - 1)
    up, down = g[hi] - y, y - g[hi - 1]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    sign = (torch.signbit(b) & ~bad[..., None]).long() << (bits - 1)
    return (code | sign).flatten(-2).to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)


def pack(code, bits):
    return code if bits == 8 else code[..., ::2] | code[..., 1::2] << 4


def unpack(packed, bits):
    return packed if bits == 8 else torch.stack([packed & 15, packed >> 4], -1).flatten(-2)


def values(code, scale, bits):
    """What codes [..., hd] and scale bytes [..., hd / 32] stand for."""
    g, low = grid(bits), code.long() & ((1 << (bits - 1)) - 1)
    v = g[low.clamp_max(len(g) - 1)] * torch.where(code.long() >> (bits - 1) > 0, -1.0, 1.0)
    s = torch.where(scale == 255, math.nan, 2.0 ** (scale.double() - 127))
    return v * s.repeat_interleave(32, -1)


def rounded(v, bits):
    return values(*quantize(v, bits), bits)


def attention(q, k, v, seen):
    """q [n][hd], k, v [m][hd], seen [n][m], float64: the weighted means (zeros for a row that sees nothing) and how far a
    kernel that rounds the probabilities and the result to bf16 and computes in fp32 may be off, element by element:
      probabilities: half a step of bf16, and the error e of their exponents, on all of them and on their sum (which may be taken
      before or after the rounding);
      e: a dot product of hd terms in fp32, its scaling, the exponential (1 unit in 2^22), next to scores of size s;
      sums over m terms in fp32; the result: half a step of bf16;
      fp32 ends at 2^-126: a probability (relative to the largest, which is 1, so the sum is at least 1), a share's weight or a
      product below it may become 0, which takes at most 2^-126 (|v| + 1) from a term, once for each of the three."""
    hd = q.shape[-1]
    s = q @ k.T / math.sqrt(hd)
    size = (q.abs() @ k.abs().T / math.sqrt(hd)).masked_fill(~seen, 0.0).amax(-1, keepdim=True) if k.shape[0] else torch.zeros(q.shape[0], 1)
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_min(-1e300) if k.shape[0] else torch.zeros(q.shape[0], 1).double()
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / total.masked_fill(total == 0, 1.0)
    vz = torch.nan_to_num(v, 0.0, 0.0, 0.0)
    o = p @ vz
    unit = 2.0 ** -24
    e = (hd + 4) * unit * size + 3 * unit * size + 2.0 ** -22
    off = (2 * HALF_BF16 + 2 * e + 2 * k.shape[0] * unit) * (p @ vz.abs())
    off = off + 3 * 2.0 ** -126 * (vz.abs() + 1).sum(0)
    return o, off + HALF_BF16 * (o.abs() + off)
