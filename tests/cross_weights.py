"""Bounds of cross attention of up to 16 rows per key/value head (Nq * Hq / Hkv).

A weight is held as two bf16 numbers that add up to it: the second is the rounding of what the first
leaves, at most 2^-8 of it, so the two are off by 2^-16 of the weight (half a step is 2^-8 of a
value).  In window_reference's bound, 2^-8 sum w |v| for the weights becomes 2^-16 sum w |v|."""
import math

import torch

import window_reference as ref


def cross64(q, k, v, mask=None):
    """o, lse and their bounds, all heads; mask [B, Nk]."""
    q, k, v = (t.cpu().double() for t in (q, k, v))
    B, Hq, Nq, D = q.shape
    share = Hq // k.shape[1]
    o, ob = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(B, Hq, Nq, dtype=torch.float64)
    lb = torch.empty_like(lse)
    for b in range(B):
        at = torch.arange(k.shape[2])
        if mask is not None:
            at = at[mask[b].cpu()]
        see = torch.ones(Nq, len(at), dtype=torch.bool)
        for h in range(Hq):
            x = v[b, h // share][at]
            o[b, h], lse[b, h], ob[b, h], lb[b, h] = ref.attend(
                q[b, h], k[b, h // share][at], x, see, D ** -0.5, vround=x.abs() * ref.HALF)
    return o, lse, ob, lb


def rounded(q, k, v, parts):
    """o in 64 bits but for the weights against the row's largest, held in `parts` bf16 numbers, and
    for the result, rounded to bf16."""
    q, k, v = (t.double() for t in (q, k, v))
    share = q.shape[1] // k.shape[1]
    k, v = (t.repeat_interleave(share, 1) for t in (k, v))
    x = q @ k.transpose(2, 3) / math.sqrt(q.shape[-1])
    p = torch.exp(x - x.amax(-1, keepdim=True))
    held, rest = torch.zeros_like(p), p
    for _ in range(parts):
        held = held + rest.bfloat16().double()
        rest = p - held
    return ((held @ v) / p.sum(-1, keepdim=True)).bfloat16()


def inputs(seed, B, Hq, Hkv, Nq, Nk, D):
    """Scores of a few units, so that several keys share a row's weight."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(B, Hq, Nq, D, generator=g).bfloat16()
    k, v = (torch.randn(B, Hkv, Nk, D, generator=g).bfloat16() for _ in range(2))
    return q, k, v
