"""What window attention and attention over the quantised cache may be off by, as sizes of errors
instead of limits, for many rows at a time (torch on the CPU, 64 bits).  window_reference has
limits, which single values are held to; they are far wider than the errors.

lse: nothing but fp32 sums is rounded.  A score is a sum of terms t_d: q_d k_d for bf16 rows; q_d s u_d
and q_d m for the cache, whose codes u, steps s and smallest values m all enter exactly.  An fp32
addition is off by at most 2^-23 of the partial sum (truncating ones too), the partial sums of terms
of either sign are of the size of ||t||, and the errors of D additions add up like independent ones:
sqrt(D) 2^-23 ||t||, times the scale.  lse takes the mean of the scores' errors, weighted by the
softmax (independence between keys is given no credit).  Its own roundings, 2^-24 each: the scale to
fp32 and times log2(e) (2), the weights' arguments (1), log2 (2), the reference added (1), ln 2 and
its product (2), of a value of up to |lse| + log(keys).  The normaliser is summed 64 keys at a time,
after at most 16 additions among them: sqrt(keys / 64 + 16) 2^-23.

o: the weights w are rounded before they meet V, independently of each other, to bf16 (half a step,
2^-8, of w s u; of w v where V is bf16 rows) or, with more than 32 rows per key/value head, to fp16
like V (2^-11 of w v, twice): that times the root of the sum of squares over the keys.  The fp16
weights are 2^7 and more at a row's largest, V 2^14 at its largest, and what lies below fp16's normal
range is off by up to 2^-25: 2^-32 max |v| a key, as independently.  The result is rounded to bf16:
2^-8 |o|.  The weights' errors are lse's and the scores': two sizes, times sum
w |v|.  The fp32 sums: sqrt(keys) 2^-23 of sum w |v|, and of w s (16 + u) and w s 16 where 4-bit
codes enter as 16 + u.

The root mean square of error / size over the values has to be at most 1, and no single one above 4."""
import math

import torch

import window_reference as ref

STEP, HALF, HALF16 = 2.0 ** -23, 2.0 ** -8, 2.0 ** -11


def attend(q, k, v, terms2, mask, scale, rounded, summed, fp16=False):
    """One head: q [n, D], k, v [L, D] float64 where mask [n, L]; terms2 [n, L]: ||t||^2; rounded
    [L, D]: what a rounded weight multiplies, times half a step; summed [L, D]: magnitudes of what
    is summed to o; fp16: weights and V are.  Returns lse, its size, o, its size."""
    x = ((q @ k.t()) * scale).masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(x, 1)
    w = torch.exp(x - lse[:, None])
    D, cnt = q.shape[1], mask.sum(1).double()
    size = (w * terms2.clamp(min=0).sqrt()).sum(1) * (scale * math.sqrt(D) * STEP)
    size += 8 * STEP / 2 * (lse.abs() + cnt.log()) + (cnt / 64 + 16).sqrt() * STEP
    o = w @ v
    osize = (w ** 2 @ rounded ** 2).sqrt() + HALF * o.abs() + 2 * size[:, None] * (w @ v.abs())
    osize += cnt.sqrt()[:, None] * STEP * (w @ summed) + 1e-30
    if fp16:
        osize += cnt.sqrt()[:, None] * 2.0 ** -32 * v[mask.any(0)].abs().max()
    return lse, size, o, osize


def window_attn(q, k, v, window, sinks, causal, scale=0.0):
    q, k, v = q.cpu().double(), k.cpu().double(), v.cpu().double()
    (B, Hq, Nq, D), (_, Hkv, Nk, _) = q.shape, k.shape
    scale = scale or D ** -0.5
    mask = ref.sees(torch.arange(Nq) + Nk - Nq, torch.arange(Nk), window, sinks, causal, Nk)
    out = []
    for b in range(B):
        for h in range(Hq):
            kk, vv = k[b, h // (Hq // Hkv)], v[b, h // (Hq // Hkv)]
            out.append(attend(q[b, h], kk, vv, q[b, h] ** 2 @ (kk ** 2).t(), mask, scale,
                              HALF * vv.abs(), vv.abs()))
    return tuple(torch.stack(x).unflatten(0, (B, Hq)) for x in zip(*out))


def cache_attn(q, k, v, bits, lens, window=1 << 30, sinks=0, scale=0.0, k_as=None, v_mask=255):
    """q [B, Hq, n, D]; k, v lists of [Hkv, lens[b], D] bf16.  k_as: a type that K's held values go
    through, v_mask: bits of V's codes that count (planted mistakes)."""
    q = q.cpu().double()
    B, Hq, n, D = q.shape
    scale = scale or D ** -0.5
    out = []
    for b, L in enumerate(lens):
        mask = ref.sees(torch.arange(n) + L - n, torch.arange(L), window, sinks, True, L)
        group = Hq // k[b].shape[0]
        many = n * group > 32
        for g in range(k[b].shape[0]):
            u, m, s = ref.quantise(k[b][g].cpu(), bits)
            su, m = ref.spread(s) * u.view(L, D), ref.spread(m)
            kk = m + su if k_as is None else (m + su).to(k_as).double()
            vu, vm, vs = ref.quantise(v[b][g].cpu(), bits)
            vu, vm, vs = (vu.long() & v_mask).view(L, D), ref.spread(vm), ref.spread(vs)
            vv = vm + vs * vu
            rounded = 2 * HALF16 * vv.abs() if many else HALF * vs * vu
            summed = vv.abs() if many else vm.abs() + vs * (vu + (32 if bits == 4 else 0))
            for h in range(g * group, (g + 1) * group):
                out.append(attend(q[b, h], kk, vv, q[b, h] ** 2 @ (su ** 2 + m ** 2).t(), mask,
                                  scale, rounded, summed, many))
    return tuple(torch.stack(x).unflatten(0, (B, Hq)) for x in zip(*out))


def misses(got, exact, size):
    """By how much values are past their sizes: at most 1 passes."""
    r = (got.cpu().double() - exact).abs() / size
    return max(float((r * r).mean().sqrt()), float(r.max()) / 4)


# ---- inputs, shared by the tests on the GPU and of the bounds ----

def rows(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).bfloat16()


# The second scale gives a row few keys, so that nothing averages a score's error away.
SCALES = {"many keys": 1.0, "few keys": 8.0}
LENS = [2000, 1500, 777, 1801]
# Rows per key/value head: 4, 12, 30, 96 and 160.
ROWS = [(1, 4), (2, 6), (5, 6), (12, 8), (20, 8)]
WINDOWS = [(None, 0), (1000, 37)]


def cache_case(n, Hq, D, which):
    """q, the sequences' K and V, and the softmax scale.  K lies away from 0, where m + s u has more
    bits than fp16 (s is that much smaller than m)."""
    q = rows(n, len(LENS), Hq, n, D) * 1.5
    ks = [rows(100 + b, 1, L, D) / 2 + rows(99, 1, 1, D) / 4 + 2.5 for b, L in enumerate(LENS)]
    vs = [rows(200 + b, 1, L, D) for b, L in enumerate(LENS)]
    return q, ks, vs, SCALES[which] / math.sqrt(D)


def window_case(D, which):
    q, k, v = rows(1, 2, 2, 700, D) * 1.5, rows(2, 2, 1, 700, D) / 2 + 2.5, rows(3, 2, 1, 700, D)
    return q, k, v, SCALES[which] / math.sqrt(D)
