"""Plain 64-bit forms of window attention, of the quantised cache's format and of attention over
it, with error bounds derived from the kernels' arithmetic (torch on the CPU).

Bounds.  A bf16 rounding is off by at most 2^-8 of the value (half a step).  The kernels round
the softmax weights (times the step s of the cache's format) to bf16 for the product with V, and
the result once more; everything else is fp32.  With w the exact weights of a row (sum 1):
  |o - o_ref| <= 2^-8 sum_j w_j |x_j| + 2^-8 |o_ref| + 2 e sum_j w_j |v_j| + tiny,
x_j = v_j (bf16 rows) or s_j u_j = v_j - m_j (the cache), and e the error of a score (a weight's
relative error is about e, and the normaliser's again).  A score of D products accumulated in
fp32 is off by at most (D + 8) 2^-23 of the sum of its terms' magnitudes (2^-23 a step, so that
truncating additions are covered too); the cache's 4-bit codes enter as 16 + u, so their terms
are |q| s (16 + u) and 16 |q| s.  Calls of more than 32 rows per key/value head take V's values and
the weights rounded to fp16 (half a step: 2^-11; scaled by powers of two so that what lies below its
normal range is under 2^-29 of the largest): 2 * 2^-11 sum_j w_j |v_j| in place of 2^-8 sum_j w_j
|x_j|.  The sums over keys add n 2^-23 of theirs.  lse is off by e, the
normaliser's n 2^-23 and four ulps of its own fp32 value."""
import math

import torch

HALF = 2.0 ** -8
HALF16 = 2.0 ** -11
STEP = 2.0 ** -23
GROUP = 64


def quantise(x, bits):
    """(codes, m, s) of bf16 rows [..., D]: codes [..., D], m and s [..., D / 64], in the fp32
    steps that the format is defined by, as float64."""
    M = float(2 ** bits - 1)
    t = x.float().unflatten(-1, (-1, GROUP))
    bad = ~torch.isfinite(t).all(-1)
    t = torch.where(bad[..., None], torch.zeros_like(t), t)
    m, top = t.amin(-1), t.amax(-1)
    bad |= ~torch.isfinite(top - m)
    s = ((top - m) / M).bfloat16().float()
    s = torch.where((s < 2.0 ** -100) | bad, torch.zeros_like(s), s)
    safe = torch.where(s == 0, torch.ones_like(s), s)[..., None]
    u = torch.round((t - m[..., None]) / safe).clamp(max=M)
    u = torch.where(s[..., None] == 0, torch.zeros_like(u), u)
    nan = torch.full_like(m, math.nan)
    m, s = torch.where(bad, nan, m), torch.where(bad, nan, s)
    return u.double().flatten(-2), m.double(), s.double()


def spread(p):
    return p.repeat_interleave(GROUP, -1)


def held(x, bits):
    """What the cache stands for, float64 (exact: a bf16 plus a product of 16 bits)."""
    u, m, s = quantise(x, bits)
    return spread(m) + spread(s) * u


def sees(p, j, window, sinks, causal, L):
    p, j = p[:, None], j[None, :]
    near = (j > p - window) & (torch.ones_like(p, dtype=torch.bool) if causal else j < p + window)
    return (near | (j < sinks)) & (j < L) & ((j <= p) if causal else torch.ones_like(near))


def attend(q, k, v, mask, scale, kmag=None, vmag=None, vround=None, fp16=False):
    """One head: q [n, D], k, v [L, D] float64 where mask [n, L].  Returns o, lse and their
    bounds.  kmag, vmag: magnitudes that enter the fp32 sums in place of |k|, |v|; vround: what
    the rounded weights multiply."""
    n, D = q.shape
    kmag = k.abs() if kmag is None else kmag
    vmag = v.abs() if vmag is None else vmag
    vround = v.abs() if vround is None else vround
    any_seen = mask.any(0)
    k, v, kmag, vmag, vround = (torch.where(any_seen[:, None], t, torch.zeros_like(t))
                                for t in (k, v, kmag, vmag, vround))
    x = (q @ k.t()) * scale
    x = x.masked_fill(~mask, -math.inf)
    err = ((q.abs() @ kmag.t()) * scale * (D + 8) * STEP).masked_fill(~mask, 0.0)
    e = err.amax(1, keepdim=True) if mask.shape[1] else torch.zeros(n, 1, dtype=torch.float64)
    lse = torch.logsumexp(x, 1)
    w = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    o = w @ v
    cnt = mask.sum(1, keepdim=True).double()
    rounded = 2 * HALF16 * (w @ v.abs()) if fp16 else HALF * (w @ vround)
    bound = (rounded * (1 + HALF) + HALF * o.abs() * (1 + 2 * HALF)
             + (2 * e + (cnt + 16) * STEP) * (w @ vmag) + 1e-30)
    finite = torch.where(torch.isfinite(lse), lse.abs(), torch.zeros_like(lse))
    lse_bound = e[:, 0] + (cnt[:, 0] + 8) * STEP + 8 * STEP * finite
    return o, lse, bound, lse_bound


def window_attn(q, k, v, window, sinks, causal, lens=None, scale=0.0):
    """All heads; rows at or past lens are NaN (to be left out)."""
    q, k, v = (t.cpu().double() for t in (q, k, v))
    B, Hq, Nq, D = q.shape
    Hkv, Nk = k.shape[1:3]
    scale = scale or D ** -0.5
    o = torch.full_like(q, math.nan)
    ob = torch.zeros_like(q)
    lse = torch.full((B, Hq, Nq), math.nan, dtype=torch.float64)
    lb = torch.zeros_like(lse)
    for b in range(B):
        L = Nk if lens is None else min(max(int(lens[b]), 0), Nk)
        n = min(Nq, max(0, L - (Nk - Nq)))
        if n == 0:
            continue
        p = torch.arange(n) + Nk - Nq
        mask = sees(p, torch.arange(L), window, sinks, causal, L)
        for h in range(Hq):
            kk, vv = k[b, h // (Hq // Hkv), :L], v[b, h // (Hq // Hkv), :L]
            o[b, h, :n], lse[b, h, :n], ob[b, h, :n], lb[b, h, :n] = attend(q[b, h, :n], kk, vv,
                                                                           mask, scale)
    return o, lse, ob, lb


def cache_attn(q, k, v, bits, lens, n_new=None, window=1 << 30, sinks=0, scale=0.0, hidden=None):
    """q [B, Hq, n, D] over the sequences' rows: k, v lists of [Hkv, lens[b], D] bf16 (as they
    were before they were cached).  hidden[b]: bool [lens[b]], tokens that no page holds.  Rows at
    or past n_new are NaN."""
    q = q.cpu().double()
    B, Hq, n, D = q.shape
    scale = scale or D ** -0.5
    o = torch.full_like(q, math.nan)
    ob = torch.zeros_like(q)
    lse = torch.full((B, Hq, n), math.nan, dtype=torch.float64)
    lb = torch.zeros_like(lse)
    for b in range(B):
        L = int(lens[b])
        nb = n if n_new is None else min(max(int(n_new[b]), 0), n)
        if nb == 0:
            continue
        p = torch.arange(nb) + L - nb
        mask = sees(p, torch.arange(L), window, sinks, True, L)
        if hidden is not None:
            mask &= ~hidden[b][None, :]
        Hkv = k[b].shape[0]
        off = 16.0 if bits == 4 else 0.0
        for g in range(Hkv):
            ku, km, ks = quantise(k[b][g].cpu(), bits)
            vu, vm, vs = quantise(v[b][g].cpu(), bits)
            ku, vu = ku.reshape(L, D), vu.reshape(L, D)
            kk, vv = spread(km) + spread(ks) * ku, spread(vm) + spread(vs) * vu
            kmag = spread(km).abs() + spread(ks) * (ku + 2 * off)
            vmag = spread(vm).abs() + spread(vs) * (vu + 2 * off)
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                r = attend(q[b, h, :nb], kk, vv, mask, scale, kmag, vmag, spread(vs) * vu,
                           fp16=n * (Hq // Hkv) > 32)
                o[b, h, :nb], lse[b, h, :nb], ob[b, h, :nb], lb[b, h, :nb] = r
    return o, lse, ob, lb


def check(o, lse, ref, label=""):
    """The kernel's outputs against a reference's; rows that are NaN there are left out."""
    ro, rl, ob, lb = ref
    rows = ~torch.isnan(rl)
    o, lse = o.cpu().double(), lse.cpu().double()
    assert torch.isfinite(o[rows]).all(), label
    err = (o - ro).abs()[rows] - ob[rows]
    if err.numel():
        assert err.max() <= 0, f"{label}: o past its bound by {err.max():.3e}"
    empty = rows & (rl == -math.inf)
    assert torch.equal((lse == -math.inf) & rows, empty), label
    assert (o[empty] == 0).all(), label
    some = rows & ~empty
    err = (lse - rl).abs()[some] - lb[some]
    if err.numel():
        assert err.max() <= 0, f"{label}: lse past its bound by {err.max():.3e}"
