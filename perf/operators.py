"""Attention with a sliding window and sinks, the quantised key/value cache, and attention over
it, as measurable cases.

A case is one call, or the calls a model's layer makes together:

  window  attention of a prompt with a sliding window and a few first tokens that stay visible
  store   a prompt's K and V quantised into the paged cache and read back
  read    a cached prompt read back as bf16 (for a selection over it)
  attn    attention of new tokens over the cache
  step    a decoding step: the new tokens' K and V written, then attention over the cache

With ``own`` the calls go to the library's entry points; without it the same operators are
computed from elementary torch operations, with the cache held as whole bytes (one code each).

The cache holds groups of 64 values of one token and head: the smallest value m (bf16), a step s
(bf16, the range over 2^bits - 1) and codes u; a value stands for m + s u.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 64      # values that share a step and a smallest value
ALL = 1 << 30   # a window that hides nothing


def listed():
    return [
        # The first tokens after a short prompt, one user: latency of a decoding step.
        dict(name="step_1x700", kind="step", B=1, Hq=28, Hkv=4, D=128, bits=4, page=64, lo=700,
             hi=700, n=1, window=ALL, sinks=0),
        # A server's step over 64 conversations of very different lengths, grouped heads.
        dict(name="step_64x8k", kind="step", B=64, Hq=32, Hkv=8, D=128, bits=4, page=64, lo=37,
             hi=8192, n=1, window=ALL, sinks=0),
        # Long video prompts, a token each: the cache is what is read.
        dict(name="attn_4x131k", kind="attn", B=4, Hq=28, Hkv=4, D=128, bits=4, page=128,
             lo=131072, hi=131072, n=1, window=ALL, sinks=0),
        # Five drafted tokens per sequence checked at once, 64-wide heads, 8 bits, no shared heads.
        dict(name="attn_draft_8x6k", kind="attn", B=8, Hq=12, Hkv=12, D=64, bits=8, page=32,
             lo=1501, hi=6007, n=5, window=ALL, sinks=0),
        # The window layers of such a model: 32k tokens held, 4096 and the first 64 seen.
        dict(name="step_window_16x32k", kind="step", B=16, Hq=28, Hkv=4, D=128, bits=4, page=64,
             lo=4000, hi=32768, n=1, window=4096, sinks=64),
        # The next 512 tokens of a prompt over what is cached of it.
        dict(name="attn_chunk_33k", kind="attn", B=1, Hq=28, Hkv=4, D=128, bits=8, page=64,
             lo=33280, hi=33280, n=512, window=ALL, sinks=0),
        # A padded batch of short prompts in a window layer, 64-wide heads.
        dict(name="window_2x1k", kind="window", B=2, Hq=16, Hkv=4, D=64, lo=611, hi=1000, Nq=1000,
             Nk=1000, window=128, sinks=4, causal=True),
        # Causal prefill of a vision-language model, 32k tokens, a window of 4096.
        dict(name="window_vlm_32k", kind="window", B=1, Hq=28, Hkv=4, D=128, lo=32768, hi=32768,
             Nq=32768, Nk=32768, window=4096, sinks=16, causal=True),
        # The 75k-token video DiT layer: one latent frame (3600 tokens) to either side, and the
        # first frame.
        dict(name="window_dit_75k", kind="window", B=1, Hq=40, Hkv=40, D=128, lo=75600, hi=75600,
             Nq=75600, Nk=75600, window=3600, sinks=3600, causal=False),
        # A 32k-token prompt into the cache.
        dict(name="store_32k", kind="store", B=1, Hkv=4, D=128, bits=4, page=64, lo=32768,
             hi=32768, n=32768),
        # A padded batch of short prompts into the cache, 64-wide heads, 8 bits.
        dict(name="store_16x700", kind="store", B=16, Hkv=12, D=64, bits=8, page=32, lo=90, hi=700,
             n=700),
        # A cached 131k-token prompt back to bf16.
        dict(name="read_131k", kind="read", B=1, Hkv=4, D=128, bits=4, page=128, lo=131072,
             hi=131072, n=131072),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "attn", "attn", "window", "window", "store", "read"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 4, 7, 8] if Hkv < 8 else [1, 2, 4])
    if kind == "window":
        Nk = _log(rng, 100, 75600)
        B = rng.choice([1, 1, 2, 3]) if Nk < 20000 else 1
        Nq = Nk if rng.random() < 0.7 else rng.randint(1, Nk)
        return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, lo=max(1, Nk - Nq + Nq // 2) if B > 1 else Nk,
                    hi=Nk, Nq=Nq, Nk=Nk, window=_log(rng, 16, min(Nk + 16, 6000)),
                    sinks=rng.choice([0, 1, 4, 16, 64, 1000]), causal=rng.random() < 0.6)
    bits, page = rng.choice([4, 4, 8]), rng.choice([32, 64, 64, 128])
    hi = _log(rng, 20, 131072)
    B = min(_log(rng, 1, 64), max(1, 400000 // hi))
    lo = rng.randint(max(1, hi // 20), hi)
    if kind in ("store", "read"):
        return dict(kind=kind, B=B, Hkv=Hkv, D=D, bits=bits, page=page, lo=lo, hi=hi, n=hi)
    n = rng.choice([1, 1, 1, 2, 4, 7])
    if kind == "attn" and rng.random() < 0.2:
        n, B, lo = min(hi, _log(rng, 16, 512)), 1, hi
    n = min(n, lo)
    window, sinks = ALL, 0
    if rng.random() < 0.35:
        window, sinks = _log(rng, 16, 8192), rng.choice([0, 1, 4, 64])
    return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, bits=bits, page=page, lo=lo, hi=hi, n=n,
                window=window, sinks=sinks)


def _lens(case):
    """Tokens of each sequence: spread over [lo, hi] in equal ratios, the longest last."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if b == B - 1 else int(round(lo * (hi / lo) ** (b / (B - 1)))) for b in range(B)]


def _row_bytes(case):
    """Bytes a token and head take in the cache, K and V: codes and one (m, s) per group."""
    return 2 * (case["D"] * case["bits"] // 8 + case["D"] // GROUP * 4)


def work(case):
    """Bytes: inputs read once, outputs written once (of the cache, the tokens that some row
    sees); operations: the two products over the visible pairs, or two per value converted."""
    D, Hkv, lens = case["D"], case["Hkv"], _lens(case)
    if case["kind"] in ("store", "read"):
        tokens = float(sum(lens)) * Hkv
        b = tokens * (4.0 * D + _row_bytes(case))
        return {"bytes": b + (tokens * 4.0 * D if case["kind"] == "store" else 0.0),
                "flops": 2.0 * tokens * 2 * D * (2 if case["kind"] == "store" else 1)}
    Hq, w, sinks = case["Hq"], case["window"], case["sinks"]
    pairs = rows = seen = 0.0
    for L in lens:
        if case["kind"] == "window":
            p = torch.arange(case["Nk"] - case["Nq"], L, dtype=torch.float64)
        else:
            p = torch.arange(L - case["n"], L, dtype=torch.float64)
        if p.numel() == 0:
            continue
        left = p.clamp(max=w - 1)
        right = torch.zeros_like(p)
        if not case.get("causal", True):
            right = (L - 1 - p).clamp(max=w - 1)
        far = (p - left).clamp(max=sinks)
        if not case.get("causal", True):  # sinks past the window
            far = far + (min(sinks, L) - (p + right + 1)).clamp(min=0)
        pairs += float((left + 1 + right + far).sum())
        rows += p.numel()
        first = float(p[0] - left[0])
        seen += L - first + min(first, float(sinks))
    qo = 4.0 * rows * Hq * D + 4.0 * rows * Hq
    if case["kind"] == "window":
        return {"bytes": qo + 4.0 * seen * Hkv * D, "flops": 4.0 * D * Hq * pairs}
    new = 4.0 * D * Hkv * rows if case["kind"] == "step" else 0.0
    return {"bytes": qo + seen * Hkv * _row_bytes(case) + new, "flops": 4.0 * D * Hq * pairs}


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _kv(case, g, n, u, off):
    """K and V of n tokens, [1, Hkv, n, D] bf16 as a projection leaves them (token-major rows):
    N(0, 1), channels of K with offsets of their own, the first token a sink."""
    H, D = case["Hkv"], case["D"]
    k = torch.randn(1, n, H, D, generator=g, device=DEV) + off
    v = torch.randn(1, n, H, D, generator=g, device=DEV)
    k[:, 0] += 0.7 * u
    return k.bfloat16().transpose(1, 2), v.bfloat16().transpose(1, 2)


def _queries(case, g, n, u):
    B, H, D = case["B"], case["Hq"], case["D"]
    q = torch.randn(B, n, H, D, generator=g, device=DEV)
    q += u.repeat_interleave(H // case["Hkv"], 0)
    return q.bfloat16().transpose(1, 2)


def _directions(case, g):
    u = torch.randn(case["Hkv"], case["D"], generator=g, device=DEV)
    off = torch.randn(case["Hkv"], case["D"], generator=g, device=DEV)
    return u, off


def _table(case, g):
    """Pages of the sequences, in the order in which a server that frees and takes pages comes to
    hold them (any), -1 past a sequence's last."""
    per = [-(-L // case["page"]) for L in _lens(case)]
    pages = sum(per) + 3
    ids = torch.randperm(pages, generator=g, device=DEV).int()
    table = torch.full((case["B"], max(per)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, c in enumerate(per):
        table[b, :c] = ids[at:at + c]
        at += c
    return table, pages


def _inputs(case, seed):
    """What both sides and the 64-bit form start from."""
    g = _gen(seed)
    u, off = _directions(case, g)
    lens = _lens(case)
    s = dict(lens_list=lens, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    if case["kind"] == "window":
        kv = [_kv(case, g, case["Nk"], u, off) for _ in range(case["B"])]
        s["k"], s["v"] = (torch.cat(x) if case["B"] > 1 else x[0] for x in zip(*kv))
        s["q"] = _queries(case, g, case["Nq"], u)
        return s, None
    s["table"], s["pages"] = _table(case, g)
    if case["kind"] != "store" and case["kind"] != "read":
        s["q"] = _queries(case, g, case["n"], u)
    return s, lambda b: _kv(case, g, lens[b], u, off)


def prepare(case, seed):
    s, kv = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "window":
        return s
    B, n = case["B"], case["n"]
    new = case["kind"] in ("step", "store")
    if own:
        import paper_2603_29494_amd as va
        s["cache"] = va.cache_alloc(s["pages"], case["Hkv"], case["D"], case["page"], case["bits"])
    else:
        s["cache"] = _plain_cache(case, s["pages"])
    if new:  # the rows the call writes, a padded batch
        nk = torch.zeros(B, n, case["Hkv"], case["D"], dtype=torch.bfloat16, device=DEV)
        nv = torch.zeros_like(nk)
        s["k"], s["v"] = nk.transpose(1, 2), nv.transpose(1, 2)
        s["n_new"] = torch.tensor([min(n, L) for L in s["lens_list"]], dtype=torch.int32,
                                  device=DEV)
    for b, L in enumerate(s["lens_list"]):
        k, v = kv(b)
        m = min(n, L)
        if new:
            s["k"][b, :, :m], s["v"][b, :, :m] = k[0, :, L - m:], v[0, :, L - m:]
        if case["kind"] == "store":
            continue
        if own:
            va.cache_write(s["cache"], k, v, s["table"][b:b + 1], s["lens"][b:b + 1])
        else:
            _plain_write(s["cache"], k[0], v[0], s["table"][b], 0)
    if case["kind"] in ("store", "read"):  # where a program takes the rows to
        shape = (B, case["Hkv"], max(s["lens_list"]), case["D"])
        s["out"] = tuple(torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the library's calls ----

def _run_own(s):
    import paper_2603_29494_amd as va
    c = s["case"]
    if c["kind"] == "window":
        lens = s["lens"] if c["B"] > 1 else None
        o, lse = va.window_attn(s["q"], s["k"], s["v"], c["window"], sinks=c["sinks"],
                                causal=c["causal"], lens=lens, return_lse=True)
        return {"o": o, "lse": lse}
    if c["kind"] in ("step", "store"):
        va.cache_write(s["cache"], s["k"], s["v"], s["table"], s["lens"], n_new=s["n_new"])
    if c["kind"] in ("store", "read"):
        k, v = va.cache_read(s["cache"], s["table"], s["lens"], c["n"], out=s["out"])
        return {"k": k, "v": v}
    o, lse = va.cache_attn(s["q"], s["cache"], s["table"], s["lens"], window=c["window"],
                           sinks=c["sinks"], return_lse=True)
    return {"o": o, "lse": lse}


# ---- the plain form ----

def _plain_cache(case, pages):
    H, D, page = case["Hkv"], case["D"], case["page"]
    shape = (pages, H, page)
    z = dict(device=DEV)
    return dict(page=page, bits=case["bits"],
                ku=torch.zeros(*shape, D, dtype=torch.uint8, **z),
                vu=torch.zeros(*shape, D, dtype=torch.uint8, **z),
                kp=torch.zeros(*shape, D // GROUP, 2, dtype=torch.bfloat16, **z),
                vp=torch.zeros(*shape, D // GROUP, 2, dtype=torch.bfloat16, **z))


def _quantise(x, bits):
    """Codes [..., D] and (m, s) [..., D / GROUP, 2] of bf16 rows."""
    top = float(2 ** bits - 1)
    t = x.float().unflatten(-1, (-1, GROUP))
    m = t.amin(-1, keepdim=True)
    s = ((t.amax(-1, keepdim=True) - m) / torch.tensor(top, device=x.device)).bfloat16().float()
    flat = s < 2.0 ** -100
    s = torch.where(flat, torch.zeros_like(s), s)
    u = torch.round((t - m) / torch.where(flat, torch.ones_like(s), s)).clamp(max=top)
    u = torch.where(flat, torch.zeros_like(u), u)
    return u.to(torch.uint8).flatten(-2), torch.cat([m, s], -1).bfloat16()


def _value(u, p):
    """m + s u in 32 bits, [..., D]."""
    return (p[..., 0:1].float() + p[..., 1:2].float() * u.float().unflatten(-1, (-1, GROUP))).flatten(-2)


def _plain_write(cache, k, v, row, start):
    """Rows of one sequence ([Hkv, n, D]) at positions start, start + 1, ..."""
    at = start + torch.arange(k.shape[1], device=DEV)
    page, off = row[at // cache["page"]].long(), at % cache["page"]
    for x, u, p in ((k, "ku", "kp"), (v, "vu", "vp")):
        codes, par = _quantise(x.transpose(0, 1).contiguous(), cache["bits"])
        cache[u][page, :, off] = codes
        cache[p][page, :, off] = par


def _plain_rows(cache, row, L, name):
    """The first L tokens of one sequence as 32-bit values [Hkv, L, D]."""
    ids = row[:-(-L // cache["page"])].long()
    x = _value(cache[name + "u"][ids], cache[name + "p"][ids])
    return x.transpose(0, 1).flatten(1, 2)[:, :L]


def _attend(q, k, v, mask, grp):
    """One block of rows: q [Hq, n, D] against k, v [Hkv, m, D] where mask [n, m] holds."""
    Hq, n, D = q.shape
    s = torch.bmm(q.reshape(-1, grp * n, D), k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
    s = s.view(-1, grp, n, k.shape[1]).masked_fill_(~mask, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    l = e.sum(-1, keepdim=True)
    o = torch.bmm(e.view(-1, grp * n, k.shape[1]), v).view(-1, grp, n, D)
    o = o / torch.where(l == 0, torch.ones_like(l), l)
    return o.reshape(Hq, n, D), (top + torch.log(l)).view(Hq, n)


def _visible(p, j, case):
    w, sinks = case["window"], case["sinks"]
    p, j = p[:, None], j[None, :]
    near, first = j > p - w, j < sinks
    if case.get("causal", True):
        return (near | first) & (j <= p)
    return (near & (j < p + w)) | first


def _windowed(q, k, v, p0, case, step):
    """Rows at positions p0, p0 + 1, ... of q [Hq, n, D] against keys 0 .. L - 1, `step` rows at
    a time, against the keys that one of them sees."""
    L, n, grp = k.shape[1], q.shape[1], q.shape[0] // k.shape[0]
    w, sinks = case["window"], case["sinks"]
    out = []
    for a in range(0, n, step):
        z = min(n, a + step)
        lo = max(0, p0 + a - w + 1)
        hi = p0 + z
        if not case.get("causal", True):
            hi = min(L, max(p0 + z - 1 + w, sinks))
        first = min(sinks, lo)
        j = torch.arange(lo, hi, device=DEV)
        kk, vv = k[:, lo:hi], v[:, lo:hi]
        if first:
            j = torch.cat([torch.arange(first, device=DEV), j])
            kk, vv = torch.cat([k[:, :first], kk], 1), torch.cat([v[:, :first], vv], 1)
        p = torch.arange(p0 + a, p0 + z, device=DEV)
        out.append(_attend(q[:, a:z], kk, vv, _visible(p, j, case), grp))
    return torch.cat([x[0] for x in out], 1), torch.cat([x[1] for x in out], 1)


def _rows_at_once(case, keys):
    """Rows whose scores take about a gigabyte in 32 bits."""
    return max(1, min(1024, int(2 ** 28 // max(1, case["Hq"] * keys))))


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "window":
        q, k, v = s["q"], s["k"], s["v"]
        o = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
        lse = torch.zeros(q.shape[:3], dtype=torch.float32, device=DEV)
        p0 = c["Nk"] - c["Nq"]
        for b, L in enumerate(s["lens_list"]):
            n = L - p0
            if n <= 0:
                continue
            ob, lb = _windowed(q[b, :, :n].float(), k[b, :, :L].float(), v[b, :, :L].float(), p0,
                               c, _rows_at_once(c, min(L, 2 * c["window"] + c["sinks"])))
            o[b, :, :n], lse[b, :, :n] = ob.bfloat16(), lb
        return {"o": o, "lse": lse}
    lens, table, cache = s["lens_list"], s["table"], s["cache"]
    if c["kind"] in ("step", "store"):
        for b, L in enumerate(lens):
            m = min(c["n"], L)
            _plain_write(cache, s["k"][b, :, :m], s["v"][b, :, :m], table[b], L - m)
    if c["kind"] in ("store", "read"):
        for b, L in enumerate(lens):
            for out, name in zip(s["out"], "kv"):
                out[b, :, :L] = _plain_rows(cache, table[b], L, name).bfloat16()
        return {"k": s["out"][0], "v": s["out"][1]}
    q, n = s["q"], c["n"]
    o = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=DEV)
    for b, L in enumerate(lens):
        k, v = _plain_rows(cache, table[b], L, "k"), _plain_rows(cache, table[b], L, "v")
        ob, lse[b] = _windowed(q[b].float(), k, v, L - n, c,
                               _rows_at_once(c, min(L, c["window"] + c["sinks"])))
        o[b] = ob.bfloat16()
    return {"o": o, "lse": lse}


# ---- in 64 bits ----

def _held64(x, bits):
    """What the cache holds of bf16 rows [H, n, D], in 64 bits: the format's smallest value and
    step (rounded to bf16 from the 32-bit quotient of a 32-bit range, as the format says), codes
    from 64-bit quotients."""
    M = 2 ** bits - 1
    H, n, D = x.shape
    t = x.double().reshape(H, n, D // GROUP, GROUP)
    small, large = t.min(-1).values, t.max(-1).values
    span = (large - small).float().double()
    step = (span / M).float().bfloat16().double()
    step[step < 2.0 ** -100] = 0.0
    safe = step.clone()
    safe[step == 0.0] = math.inf
    code = ((t - small[..., None]) / safe[..., None]).round().clamp(0, M)
    return (small[..., None] + step[..., None] * code).reshape(H, n, D)


def _rows64(q, k, v, start, case):
    """Rows at positions start, start + 1, ... of q [Hq, n, D] over all keys they may see, from
    the definition: one query head and 1024 rows at a time."""
    Hq, n, D = q.shape
    L, share = k.shape[1], Hq // k.shape[0]
    two_sided = not case.get("causal", True)
    reach, sinks = min(case["window"], L), min(case["sinks"], L)
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(Hq, n, dtype=torch.float64, device=DEV)
    every = torch.arange(L, device=DEV)
    for r0 in range(0, n, 1024):
        r1 = min(n, r0 + 1024)
        pos = torch.arange(start + r0, start + r1, device=DEV)
        some = (every > start + r0 - reach) | (every < sinks)
        some &= (every < start + r1 - 1 + reach) | (every < sinks) if two_sided else every < start + r1
        at = every[some]
        gap = at.unsqueeze(0) - pos.unsqueeze(1)
        hidden = (gap.abs() >= reach) & (at < sinks).logical_not().unsqueeze(0)
        if not two_sided:
            hidden |= gap > 0
        for h in range(Hq):
            kh, vh = k[h // share][at].double(), v[h // share][at].double()
            x = (q[h, r0:r1].double() @ kh.t().contiguous()) / math.sqrt(D)
            x[hidden] = -math.inf
            lse[h, r0:r1] = x.logsumexp(1)
            o[h, r0:r1] = x.softmax(1) @ vh
    return o, lse


def exact(case, seed):
    s, kv = _inputs(case, seed)
    lens = s["lens_list"]
    if case["kind"] == "window":
        q, k, v = s["q"], s["k"], s["v"]
        o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros(q.shape[:3], dtype=torch.float64, device=DEV)
        p0 = case["Nk"] - case["Nq"]
        for b, L in enumerate(lens):
            n = L - p0
            if n > 0:
                o[b, :, :n], lse[b, :, :n] = _rows64(q[b, :, :n], k[b, :, :L], v[b, :, :L], p0,
                                                     case)
        return {"o": o, "lse": lse}
    if case["kind"] in ("store", "read"):
        k = torch.zeros(case["B"], case["Hkv"], max(lens), case["D"], dtype=torch.float64,
                        device=DEV)
        v = torch.zeros_like(k)
        for b, L in enumerate(lens):
            kb, vb = kv(b)
            k[b, :, :L], v[b, :, :L] = _held64(kb[0], case["bits"]), _held64(vb[0], case["bits"])
        return {"k": k, "v": v}
    q, n = s["q"], case["n"]
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(q.shape[:3], dtype=torch.float64, device=DEV)
    for b, L in enumerate(lens):
        kb, vb = kv(b)
        o[b], lse[b] = _rows64(q[b], _held64(kb[0], case["bits"]), _held64(vb[0], case["bits"]),
                               L - n, case)
    return {"o": o, "lse": lse}
