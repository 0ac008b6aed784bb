"""Plain restatements, in 64 bits, of what include/cofie_kv.h defines: rotary
positions, the 4-bit codes of a group, and attention over a paged cache. They
share nothing with the package. Each comes with a bound on the error of a
kernel that works in fp32 with 16-bit matrix products, derived here:

unit roundoff u: 2^-8 for bf16, 2^-11 for fp16, 2^-24 for fp32.

rotary: the angle is formed to 2^-32 turns and rounded to fp32 (2^-24 of at most
  pi), cos and sin are good to 2 ulp, the amplitude and the two products and the
  sum round once each: together under 2^-20 (|x1| + |x2|) m, then u |y|.

attention: a score is a sum of D <= 128 products in fp32, error at most
  d = 2^-17 scale sum |q| |k|. Where a kernel multiplies q by 4-bit codes held
  as 128 + n (bf16) or 1024 + n (fp16) and takes the excess off afterwards, |k|
  stands for 144 s or 1040 s. Probabilities are off by 2 d and, rounded to the
  inputs' type for the second product (for 4-bit values after the product with
  their scale, for fp16 then at least 2^-25 of the largest), by u more:
  |out - o| <= u |o| + (u + 2 d + 2^-16) sum p |v|,  |lse - l| <= d + 2^-20 (1 + |l|)
"""
from __future__ import annotations

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def frequencies(rotary_dim, base, scaling="none", factor=1.0, original_len=0.0, fast=32.0, slow=1.0):
    """(f_i, m)."""
    out, m = [], 1.0
    if scaling == "base":
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    if scaling == "yarn":
        m = 0.1 * math.log(factor) + 1.0
    for i in range(rotary_dim // 2):
        f = base ** (-2.0 * i / rotary_dim)
        if scaling == "linear":
            f /= factor
        elif scaling == "yarn":
            r = original_len * f / (2.0 * math.pi)
            g = min(1.0, max(0.0, (r - slow) / (fast - slow)))
            f = (1.0 - g) * f / factor + g * f
        out.append(f)
    return out, m


def rotate(x, positions, freq, m, layout, axes=None, back=False):
    """x [tokens, heads, d] -> (y, bound without u |y|), fp64; positions [axes, tokens] int."""
    x = x.detach().double().cpu()
    pos = positions.cpu().double().reshape(-1, x.shape[0])
    half = len(freq)
    y, slack = x.clone(), torch.zeros_like(x)
    for i, f in enumerate(freq):
        a = pos[axes[i] if axes else 0] * f
        c, s = torch.cos(a)[:, None] * m, torch.sin(a)[:, None] * (-m if back else m)
        p, r = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        y[..., p] = x[..., p] * c - x[..., r] * s
        y[..., r] = x[..., r] * c + x[..., p] * s
        slack[..., p] = slack[..., r] = 2.0 ** -20 * m * (x[..., p].abs() + x[..., r].abs())
    return y, slack


def quantise(x):
    """x [..., d] -> (codes [..., d] int, scale [..., d/64], zero [..., d/64]) by the definition, fp64."""
    y = x.detach().double().cpu().unflatten(-1, (-1, 64))
    lo, hi = y.amin(-1).clamp(max=0.0), y.amax(-1).clamp(min=0.0)
    mant, exp = torch.frexp((hi - lo) / 15.0)
    s = torch.ldexp(torch.ceil(mant * 16.0) / 16.0, exp)
    s = torch.where((hi - lo) / 15.0 < 2.0 ** -100, 0.0, s)
    u = torch.where(s > 0, s, 1.0)
    near = lambda v: torch.sign(v) * torch.floor(v.abs() + 0.5)  # noqa: E731
    zero = torch.where(s > 0, near(-lo / u).clamp(0, 15), 0.0)
    n = torch.where((s > 0)[..., None], (near(y / u[..., None]) + zero[..., None]).clamp(0, 15), 0.0)
    return n.flatten(-2).int(), s, zero.int()


def pack(codes, scale, zero):
    """Bytes and words of codes, as the pages hold them."""
    b = (codes[..., 0::2] | codes[..., 1::2] << 4).to(torch.uint8)
    w = scale.to(torch.float32).view(torch.int32) >> 16 | zero
    return b, torch.where(w >= 32768, w - 65536, w).to(torch.int16)


def unpack(codes, words):
    """(values fp64, scale per value) of bytes and words."""
    c = codes.cpu().int()
    n = torch.stack([c & 15, c >> 4], -1).flatten(-2).unflatten(-1, (-1, 64))
    w = words.cpu().int() & 0xFFFF
    s = ((w & 0xFFF0) << 16).view(torch.float32).double()[..., None]
    return ((n - (w & 15)[..., None]).double() * s).flatten(-2), s.expand(n.shape).flatten(-2)


def attend(q, k, v, visible, scale, dtype, excess=None):
    """q [n, H, d], k and v [m, H_kv, d], visible [n, m] bool -> (out, lse, bound of out, bound of lse), fp64.
    excess [m, H_kv, d]: what stands for |k| in the scores' error."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    visible = visible.cpu()
    n, H, d = q.shape
    G = H // k.shape[1]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    held = visible.any(0)[:, None, None]
    k, v = torch.where(held, k, 0.0), torch.where(held, v, 0.0)  # what nothing sees does not matter
    x = torch.einsum("nhd,mhd->hnm", q, k) * scale
    x = torch.where(visible, x, -math.inf)
    top = x.amax(-1, keepdim=True) if x.shape[-1] else torch.full((H, n, 1), -math.inf, dtype=torch.float64)
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1).T
    out = torch.einsum("hnm,mhd->nhd", p, v)
    size = torch.einsum("hnm,mhd->nhd", p, v.abs())
    mag = k.abs() if excess is None else torch.where(held, excess.double().cpu().repeat_interleave(G, 1), 0.0)
    dots = torch.einsum("nhd,mhd->hnm", q.abs(), mag)
    dots = torch.where(visible, dots, 0.0)
    delta = 2.0 ** -17 * scale * (dots.amax(-1).T if dots.shape[-1] else torch.zeros(n, H, dtype=torch.float64))
    u = UNIT[dtype]
    # one spacing of the smallest fp16 numbers, too
    b_out = u * out.abs() + (u + 2 * delta[..., None] + 2.0 ** -16) * size + 2.0 ** -24
    b_lse = delta + 2.0 ** -20 * (1 + torch.where(torch.isfinite(lse), lse.abs(), 0.0))
    return out, lse, b_out, b_lse
