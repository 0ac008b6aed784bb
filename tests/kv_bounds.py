"""The bound on attention's outputs for kernels that see the cache's numbers exactly, whatever the pages hold: 4-bit codes
enter the products as (n - z), or as (n - z) s, which 16-bit types hold. It is kv_oracle.attend's, with the numbers' own
sizes for 4-bit pages as for 16-bit ones, with two terms for what fp16 cannot hold and one for long sums:

queries   the kernel of few rows takes them to fp16, a power of two bringing the row's largest to [128, 256): an entry
          is off by at most 2^-21 there (half of fp16's smallest spacing, for the odd dimensions 16 times that), so by
          2^-28 of the row's largest, and a score by 2^-28 scale max|q| sum |k|
weights   for fp16 they are rounded to fp16 with the largest at 2^7 or more, so none is off by more than 2^-32 where
          u of it is less; with 4-bit values, few rows, weight times scale, at 2^10 or more of the largest scale s: off
          by 2^-35 s at most, and a value by 15 of that, where 15 s <= 9/8 (hi - lo) < 3 max |v|. Over m tokens:
          m 2^-32 max |v|.
sums      the tensor cores cut each product off at 2^-24 of the sum that it is added to, or below: over `chain` tokens
          that come to one sum chain 2^-24 sum p |v|. A sum holds at most 8192 tokens (fp16) or 65536 (bf16) in the
          kernel of many rows, an eighth of a CTA's tokens in that of few.
"""
from __future__ import annotations

import torch

from tests import kv_oracle as K


def attend(q, k, v, visible, scale, dtype, chain=None):
    """As kv_oracle.attend: (out, lse, bound of out, bound of lse). chain: the most tokens of a sum; all of them."""
    out, lse, b_out, b_lse = K.attend(q, k, v, visible, scale, dtype)
    chain = visible.shape[1] if chain is None else min(chain, visible.shape[1])
    b_out = b_out + chain * 2.0 ** -24 * K.attend(q, k, torch.as_tensor(v).abs(), visible, scale, dtype)[0]
    q, visible = q.double().cpu(), visible.cpu()
    held = visible.any(0)
    G = q.shape[1] // k.shape[1]
    if not bool(held.any()):
        return out, lse, b_out, b_lse
    k, v = k.double().cpu()[held], v.double().cpu()[held]
    size = k.abs().sum(-1).amax(0).repeat_interleave(G)  # [H]
    more = 2.0 ** -28 * scale * q.abs().amax(-1) * size  # [n, H]
    most = v.abs().amax((0, 2)).repeat_interleave(G)  # [H]
    floor = (visible.sum(1)[:, None] * 2.0 ** -32 * most)[..., None]
    weighed = torch.where(torch.isfinite(lse), most.expand_as(lse), 0.0)
    b_out = b_out + 2 * (more * weighed)[..., None]
    if dtype == torch.float16:
        b_out = b_out + floor
    return out, lse, b_out, b_lse + more


def exceeds(got, lse, want):
    """What passes its bound: (outputs, log-sum-exps), as bool tensors; want as attend() returns it. Rows that see nothing
    have 0 and -infinity and nothing else."""
    o, l, b_out, b_lse = want
    empty = l == -float("inf")
    bad = ~((got.double().cpu() - o).abs() <= b_out)
    bad = torch.where(empty[..., None], got.cpu() != 0, bad)
    return bad, torch.where(empty, lse.cpu() != -float("inf"), ~((lse.double().cpu() - l).abs() <= b_lse))
