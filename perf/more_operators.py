"""Rotary positions, eviction from the key/value cache, and cross attention, as measurable cases.

A case is one call, or the calls that a model's layer makes together:

  rope   q and k of a layer turned by their positions
  mass   the attention weight that new tokens put on each cached token, added up
  evict  the heaviest tokens of every head kept: which, then moved into pages of their own
         (and read back, which is how the outputs are seen)
  cross  attention of q over an encoder's states: another length, a mask over the keys

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


def listed():
    return [
        # A server's step: one token of 64 conversations, positions from their lengths.
        dict(name="rope_step_64", kind="rope", B=64, Hq=28, Hkv=4, N=1, D=128, rot=128,
             layout="half", axes=1, where="lens", scaling="none", transpose=False),
        # Gradients of a padded batch of short prompts, a part of 64-wide heads, long-context ramp.
        dict(name="rope_part_3x777", kind="rope", B=3, Hq=12, Hkv=12, N=777, D=64, rot=48,
             layout="interleaved", axes=1, where="lens", scaling="parts", transpose=True),
        # A vision-language prompt: text and image tokens on three axes that share a ladder.
        dict(name="rope_vlm_131k", kind="rope", B=1, Hq=28, Hkv=4, N=131072, D=128, rot=128,
             layout="half", axes=3, where="given", scaling="ntk", transpose=False),
        # The 75k-token video DiT layer: time, height and width, a ladder each.
        dict(name="rope_dit_75k", kind="rope", B=1, Hq=40, Hkv=40, N=75600, D=128, rot=128,
             layout="interleaved", axes=3, where="given", scaling="none", transpose=False),
        # A decoding step over long video prompts: weights of one token per sequence.
        dict(name="mass_4x131k", kind="mass", B=4, Hq=28, Hkv=4, D=128, bits=4, page=128,
             lo=131072, hi=131072, n=1),
        # The next 512 tokens of a prompt over what is cached of it.
        dict(name="mass_chunk_33k", kind="mass", B=1, Hq=28, Hkv=4, D=128, bits=8, page=64,
             lo=33280, hi=33280, n=512),
        # One short conversation cut to a budget, 64-wide heads, 8 bits.
        dict(name="evict_1x700", kind="evict", B=1, Hkv=12, D=64, bits=8, page=32, lo=700, hi=700,
             budget=256, sinks=4, recent=32),
        # Conversations of very different lengths, some shorter than the budget.
        dict(name="evict_64x8k", kind="evict", B=64, Hkv=8, D=128, bits=4, page=64, lo=37, hi=8192,
             budget=2048, sinks=16, recent=256),
        # Long video prompts cut to an eighth.
        dict(name="evict_4x131k", kind="evict", B=4, Hkv=4, D=128, bits=4, page=128, lo=131072,
             hi=131072, budget=16384, sinks=64, recent=1024),
        # A decoder's token over a short encoded text.
        dict(name="cross_1x257", kind="cross", B=1, Hq=12, Hkv=12, D=64, Nq=1, Nk=257, lo=257,
             q_lo=1, mask=False),
        # A decoding step of 16 sequences over up to 16k encoded tokens, some of them masked.
        dict(name="cross_step_16x16k", kind="cross", B=16, Hq=28, Hkv=4, D=128, Nq=1, Nk=16384,
             lo=0, q_lo=1, mask=True),
        # The text of the 75k-token video DiT layer.
        dict(name="cross_dit_75k", kind="cross", B=1, Hq=40, Hkv=40, D=128, Nq=75600, Nk=512,
             lo=512, q_lo=75600, mask=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "mass", "evict", "cross", "cross"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 4, 7, 8] if Hkv < 8 else [1, 2, 4])
    if kind == "rope":
        N = _log(rng, 1, 75600)
        B = min(_log(rng, 1, 64), max(1, 120000 // N))
        layout = rng.choice(["half", "interleaved"])
        rot = rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)])
        axes = rng.choice([1, 1, 3]) if rot >= 6 else 1
        return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, N=N, D=D, rot=rot, layout=layout, axes=axes,
                    where=rng.choice(["lens", "given", "start"]),
                    scaling=rng.choice(["none", "linear", "ntk", "parts"]) if rot >= 4 else "none",
                    transpose=rng.random() < 0.3)
    if kind == "cross":
        Nk = _log(rng, 1, 20000)
        if rng.random() < 0.4:
            Nq, B = rng.choice([1, 1, 2, 5]), min(_log(rng, 1, 32), max(1, 300000 // Nk))
        else:
            pairs = 75600 * 512 * 40 * 128 // (Hq * D)   # as the largest listed case
            Nq = min(_log(rng, 3, 75600), max(3, pairs // Nk))
            B = rng.choice([1, 1, 2, 3]) if 3 * Nq * Nk < pairs else 1
        return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, Nq=Nq, Nk=Nk,
                    lo=rng.randint(0, Nk) if B > 1 else Nk,
                    q_lo=rng.randint(1, Nq) if B > 1 else Nq, mask=rng.random() < 0.4)
    bits, page = rng.choice([4, 4, 8]), rng.choice([32, 64, 64, 128])
    hi = _log(rng, 20, 131072)
    B = min(_log(rng, 1, 64), max(1, 400000 // hi))
    lo = rng.randint(max(1, hi // 20), hi)
    if kind == "evict":
        budget = rng.randint(max(1, hi // 16), max(1, (3 * hi) // 4))
        return dict(kind=kind, B=B, Hkv=Hkv, D=D, bits=bits, page=page, lo=lo, hi=hi,
                    budget=budget, sinks=min(rng.choice([0, 1, 4, 64]), budget // 2),
                    recent=rng.randint(0, budget // 2))
    n = rng.choice([1, 1, 1, 2, 4, 7])
    if rng.random() < 0.25:
        n, B, lo = min(hi, _log(rng, 16, 512)), 1, hi
    return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, bits=bits, page=page, lo=lo, hi=hi,
                n=min(n, lo))


def _lens(case):
    """Tokens of each sequence: spread over [lo, hi] in equal steps, the longest last."""
    B, lo = case["B"], case["lo"]
    hi = case["Nk"] if case["kind"] == "cross" else case["hi"]
    return [hi if b == B - 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _rows_of(case):
    """Rows of q that each sequence of a cross case has."""
    B, lo, hi = case["B"], case["q_lo"], case["Nq"]
    return [hi if b == B - 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _n_new(case):
    """Rows that each sequence of a rope case has where its positions come from lengths."""
    B, N = case["B"], case["N"]
    return [N if b == B - 1 else (N + 1) // 2 + (N - (N + 1) // 2) * b // (B - 1)
            for b in range(B)]


def _half_bytes(case):
    """Bytes a token and head take in the cache, K or V: codes and one (m, s) per group."""
    return case["D"] * case["bits"] // 8 + case["D"] // GROUP * 4


SEEN = 0.75   # share of the keys that a mask leaves


def work(case):
    """Bytes: inputs read once, outputs written once; operations: six per rotated pair, the score
    product of every visible pair, both products of cross attention, a comparison per mass, two
    operations per value read back."""
    D, Hkv, B = case["D"], case["Hkv"], case["B"]
    if case["kind"] == "rope":
        rows = float(sum(_n_new(case)) if case["where"] == "lens" else B * case["N"])
        heads = case["Hq"] + Hkv
        pos = 4.0 * B * case["N"] * case["axes"] if case["where"] == "given" else 0.0
        return {"bytes": 4.0 * rows * heads * D + pos, "flops": 3.0 * rows * heads * case["rot"]}
    lens = _lens(case)
    if case["kind"] == "mass":
        n, Hq = case["n"], case["Hq"]
        pairs = float(sum(n * L - n * (n - 1) // 2 for L in lens))
        return {"bytes": sum(lens) * Hkv * (_half_bytes(case) + 8.0) + B * n * Hq * (2.0 * D + 4),
                "flops": 2.0 * D * Hq * pairs}
    if case["kind"] == "evict":
        kept = float(sum(min(case["budget"], L) for L in lens)) * Hkv
        held = float(sum(lens)) * Hkv
        return {"bytes": 4.0 * held + kept * (4.0 * _half_bytes(case) + 8.0 + 4.0 * D),
                "flops": held + kept * 4.0 * D}
    rows, Hq = _rows_of(case), case["Hq"]
    seen = SEEN if case["mask"] else 1.0
    pairs = sum(r * L for r, L in zip(rows, lens)) * seen
    return {"bytes": sum(rows) * Hq * (4.0 * D + 4) + sum(lens) * (4.0 * D * Hkv * seen
                                                                  + float(case["mask"])),
            "flops": 4.0 * D * Hq * pairs}


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _rows(g, B, H, N, D, add=None):
    """[B, H, N, D] bf16 as a projection leaves it (token-major rows)."""
    x = torch.randn(B, N, H, D, generator=g, device=DEV)
    if add is not None:
        x += add
    return x.bfloat16().transpose(1, 2)


def _kv(case, g, n, u, off):
    """K and V of n tokens, [1, Hkv, n, D]: N(0, 1), channels of K with offsets of their own, the
    first token a sink."""
    H, D = case["Hkv"], case["D"]
    k = torch.randn(1, n, H, D, generator=g, device=DEV) + off
    v = torch.randn(1, n, H, D, generator=g, device=DEV)
    k[:, 0] += 0.7 * u
    return k.bfloat16().transpose(1, 2), v.bfloat16().transpose(1, 2)


def _table(case, lens, g, pages, first):
    """Pages of the sequences, in the order in which a server that frees and takes pages comes to
    hold them (any), -1 past a sequence's last; `pages` of them from `first` on."""
    per = [-(-L // case["page"]) for L in lens]
    ids = torch.randperm(pages, generator=g, device=DEV).int() + first
    table = torch.full((len(lens), max(1, max(per))), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, c in enumerate(per):
        table[b, :c] = ids[at:at + c]
        at += c
    return table


def _count_pages(case, lens):
    return sum(-(-L // case["page"]) for L in lens) + 3


LADDER, CONTEXT, FACTOR = 10000.0, 8192, 16.0
SECTIONS = (2, 3, 3)   # eighths of the pairs that three axes take


def _sections(case):
    half = case["rot"] // 2
    if case["axes"] == 1:
        return [half]
    a, b = max(1, half * SECTIONS[0] // 8), max(1, half * SECTIONS[1] // 8)
    return [a, b, half - a - b]


def _own_ladders(case):
    """Whether each axis has a ladder of its own (the video layer's) or all share one."""
    return case["layout"] == "interleaved"


def _inputs(case, seed):
    """What both sides and the 64-bit form start from."""
    g = _gen(seed)
    B, D, Hkv = case["B"], case["D"], case["Hkv"]
    if case["kind"] == "rope":
        N = case["N"]
        s = dict(q=_rows(g, B, case["Hq"], N, D), k=_rows(g, B, Hkv, N, D))
        if case["where"] == "lens":
            s["new_list"] = _n_new(case)
            far = torch.randint(0, 131072, (B,), generator=g, device=DEV)
            s["n_new"] = _int32(s["new_list"])
            s["lens"] = (far + s["n_new"]).int()
        elif case["where"] == "given":
            if case["axes"] == 1:
                s["pos"] = torch.randint(0, 1 << 20, (1, B, N), generator=g, device=DEV).int()
            else:  # frames of 45 x 80, from any frame on
                t0 = torch.randint(0, 1000, (B, 1), generator=g, device=DEV)
                at = torch.arange(N, device=DEV)[None] + t0 * 3600
                s["pos"] = torch.stack([at // 3600, at // 80 % 45, at % 80]).int()
        else:
            s["start"] = int(torch.randint(0, 100000, (1,), generator=g, device=DEV))
        return s, None
    lens = _lens(case)
    s = dict(lens_list=lens, lens=_int32(lens))
    if case["kind"] == "cross":
        s["q"] = _rows(g, B, case["Hq"], case["Nq"], D)
        u = torch.randn(Hkv, D, generator=g, device=DEV)
        s["q"] = (s["q"].float() + u.repeat_interleave(case["Hq"] // Hkv, 0)[:, None]).bfloat16()
        s["k"], s["v"] = _rows(g, B, Hkv, case["Nk"], D), _rows(g, B, Hkv, case["Nk"], D)
        s["k"][:, :, 0] += (0.7 * u).bfloat16()
        s["rows_list"] = _rows_of(case)
        s["n_q"] = _int32(s["rows_list"])
        if case["mask"]:
            s["mask"] = torch.rand(B, case["Nk"], generator=g, device=DEV) < SEEN
        return s, None
    u = torch.randn(Hkv, D, generator=g, device=DEV)
    off = torch.randn(Hkv, D, generator=g, device=DEV)
    pages = _count_pages(case, lens)
    s["table"], s["pages"] = _table(case, lens, g, pages, 0), pages
    M = s["table"].shape[1] * case["page"]
    # What heads have put on their tokens so far: a few heavy ones, and many without any weight.
    s["mass"] = torch.exp(3.0 * torch.randn(B, Hkv, M, generator=g, device=DEV) - 6.0)
    s["mass"] *= torch.rand(B, Hkv, M, generator=g, device=DEV) < 0.9
    if case["kind"] == "evict":
        kept = [min(case["budget"], L) for L in lens]
        more = _count_pages(case, kept)
        s["to_table"] = _table(case, kept, g, more, pages)
        s["pages"] = pages + more
        return s, lambda b: _kv(case, g, lens[b], u, off)
    Hq, n = case["Hq"], case["n"]
    s["q"] = _rows(g, B, Hq, n, D, u.repeat_interleave(Hq // Hkv, 0))
    s["lse"] = torch.empty(B, Hq, n, device=DEV)
    kv = [_kv(case, g, L, u, off) for L in lens]
    for b, L in enumerate(lens):   # of the keys before they are quantised: near what is held
        k = kv[b][0][0].float().transpose(1, 2).contiguous()
        step = max(1, 2 ** 28 // (Hq * L))
        for a in range(0, n, step):
            z = min(n, a + step)
            x = torch.bmm(s["q"][b, :, a:z].float().reshape(Hkv, -1, D), k) / math.sqrt(D)
            x = x.view(Hq, z - a, L)
            late = torch.arange(L, device=DEV) > torch.arange(L - n + a, L - n + z,
                                                              device=DEV)[:, None]
            s["lse"][b, :, a:z] = torch.logsumexp(x.masked_fill_(late, -math.inf), -1)
    return s, lambda b: kv[b]


def prepare(case, seed):
    s, kv = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2603_29494_amd as va
    if case["kind"] == "rope":
        if own and case["scaling"] == "parts":
            # The case's own ladder, which ends its ramp at the last pair at the latest: the
            # library's goes on past that where two to four pairs have a ladder.
            freq, axis, factor = _ladder(case)
            s["plan"] = va.Rope(case["layout"], tuple(freq.tolist()), tuple(axis.tolist()), factor)
        elif own:
            s["plan"] = va.rope_plan(
                case["rot"], base=LADDER, layout=case["layout"],
                scaling=None if case["scaling"] == "none" else case["scaling"], factor=FACTOR,
                context=CONTEXT, sections=_sections(case), own_ladders=_own_ladders(case))
        else:
            s["plan"] = _ladder(case)
    if case["kind"] in ("rope", "cross"):
        return s
    if own:
        s["cache"] = va.cache_alloc(s["pages"], case["Hkv"], case["D"], case["page"], case["bits"])
    else:
        s["cache"] = _plain_cache(case, s["pages"])
    for b, L in enumerate(s["lens_list"]):
        k, v = kv(b)
        if own:
            va.cache_write(s["cache"], k, v, s["table"][b:b + 1], s["lens"][b:b + 1])
        else:
            _plain_write(s["cache"], k[0], v[0], s["table"][b])
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the library's calls ----

def _run_own(s):
    import paper_2603_29494_amd as va
    c = s["case"]
    if c["kind"] == "rope":
        q, k = va.rope(s["plan"], s["q"], s["k"], pos=s.get("pos"), lens=s.get("lens"),
                       n_new=s.get("n_new"), start=s.get("start", 0), transpose=c["transpose"])
        return {"q": q, "k": k}
    if c["kind"] == "mass":
        return {"mass": va.cache_mass(s["q"], s["lse"], s["cache"], s["table"], s["lens"],
                                      mass=s["mass"])}
    if c["kind"] == "evict":
        idx, kept = va.cache_keep(s["mass"], s["cache"], s["table"], s["lens"], c["budget"],
                                  sinks=c["sinks"], recent=c["recent"])
        mass = va.cache_gather(s["cache"], s["table"], idx, kept, s["to_table"], mass=s["mass"])
        k, v = va.cache_read(s["cache"], s["to_table"], kept, c["budget"])
        return {"idx": idx, "kept": kept, "mass": mass, "k": k, "v": v}
    more = c["B"] > 1
    o, lse = va.cross_attn(s["q"], s["k"], s["v"], lens=s["lens"] if more else None,
                           mask=s.get("mask"), n_q=s["n_q"] if more else None, return_lse=True)
    return {"o": o, "lse": lse}


# ---- the plain form ----

def _ladder(case):
    """Frequencies [rot / 2] in 64 bits, the axis of each, and the factor of the rotated values."""
    parts = _sections(case) if _own_ladders(case) else [case["rot"] // 2]
    freqs, factor = [], 1.0
    for half in parts:
        base = LADDER
        if case["scaling"] == "ntk" and half > 1:
            base = base * FACTOR ** (half / (half - 1.0))
        f = base ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        if case["scaling"] == "linear":
            f = f / FACTOR
        if case["scaling"] == "parts":
            def at(turns):   # the pair that makes that many turns over the context
                return half * math.log(CONTEXT / (turns * 2 * math.pi)) / math.log(LADDER)
            low = min(max(math.floor(at(32.0)), 0), half - 1)
            high = min(max(math.ceil(at(1.0)), 0), half - 1)
            i = torch.arange(half, dtype=torch.float64, device=DEV)
            ramp = ((i - low) / max(high - low, 0.001)).clamp(0.0, 1.0)
            f = f / FACTOR * ramp + f * (1.0 - ramp)
            factor = 0.1 * math.log(FACTOR) + 1.0
        freqs.append(f)
    axis = torch.cat([torch.full((n,), a, device=DEV) for a, n in enumerate(_sections(case))])
    return torch.cat(freqs), axis, factor


def _positions(s):
    """int64 [axes, B, N]"""
    c = s["case"]
    if "pos" in s:
        return s["pos"].long()
    at = torch.arange(c["N"], device=DEV)[None]
    if "lens" in s:
        at = at + (s["lens"] - s["n_new"]).long()[:, None]
    else:
        at = (at + s["start"]).expand(c["B"], -1)
    return at[None].expand(c["axes"], -1, -1)


def _turn(x, cos, sin, case):
    rot = case["rot"]
    y = x.float().clone()
    if case["layout"] == "half":
        a, b = y[..., :rot // 2].clone(), y[..., rot // 2:rot].clone()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    return y.bfloat16()


def _plain_rope(s):
    c = s["case"]
    freq, axis, factor = s["plan"]
    angle = _positions(s)[axis].permute(1, 2, 0).double() * freq   # [B, N, rot / 2]
    cos, sin = (torch.cos(angle) * factor).float(), (torch.sin(angle) * factor).float()
    if c["transpose"]:
        sin = -sin
    out = {}
    for name in ("q", "k"):
        y = _turn(s[name], cos[:, None], sin[:, None], c)
        if "new_list" in s:   # rows past a sequence's last
            gone = torch.arange(c["N"], device=DEV) >= s["n_new"][:, None]
            y = y.masked_fill(gone[:, None, :, None], 0.0)
        out[name] = y
    return out


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


def _plain_write(cache, k, v, row):
    """The rows of one sequence ([Hkv, n, D]) from its first token on."""
    at = torch.arange(k.shape[1], device=DEV)
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


def _plain_mass(s):
    c = s["case"]
    Hq, Hkv, n, D = c["Hq"], c["Hkv"], c["n"], c["D"]
    out = torch.zeros_like(s["mass"])
    for b, L in enumerate(s["lens_list"]):
        out[b, :, :L - n] = s["mass"][b, :, :L - n]
        k = _plain_rows(s["cache"], s["table"][b], L, "k").transpose(1, 2).contiguous()
        step = max(1, 2 ** 28 // (Hq * L))
        for a in range(0, n, step):
            z = min(n, a + step)
            q = s["q"][b, :, a:z].float().reshape(Hkv, -1, D)
            x = torch.bmm(q, k) * (1.0 / math.sqrt(D))
            w = torch.exp(x - s["lse"][b, :, a:z].reshape(Hkv, -1, 1)).view(Hkv, -1, z - a, L)
            late = torch.arange(L, device=DEV) > torch.arange(L - n + a, L - n + z,
                                                              device=DEV)[:, None]
            out[b, :, :L] += w.masked_fill_(late, 0.0).sum((1, 2))
    return {"mass": out}


def _plain_evict(s):
    c, cache = s["case"], s["cache"]
    B, H, D, budget, page = c["B"], c["Hkv"], c["D"], c["budget"], c["page"]
    z = dict(device=DEV)
    idx = torch.full((B, H, budget), -1, dtype=torch.int32, **z)
    kept = torch.zeros(B, dtype=torch.int32, **z)
    mass = torch.zeros(B, H, budget, **z)
    k, v = (torch.zeros(B, H, budget, D, dtype=torch.bfloat16, **z) for _ in range(2))
    heads = torch.arange(H, device=DEV)[:, None]
    for b, L in enumerate(s["lens_list"]):
        n = min(budget, L)
        rank = s["mass"][b, :, :L].clone()
        rank[:, :c["sinks"]] = math.inf
        rank[:, max(0, L - c["recent"]):] = math.inf
        order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :n]
        at = torch.sort(order, dim=1).values
        idx[b, :, :n] = at.int()
        kept[b] = n
        mass[b, :, :n] = s["mass"][b].gather(1, at)
        to = torch.arange(n, device=DEV)
        src = (s["table"][b].long()[at // page], heads, at % page)
        dst = (s["to_table"][b].long()[to // page][None], heads, (to % page)[None])
        for name in ("ku", "kp", "vu", "vp"):
            cache[name][dst] = cache[name][src]
        k[b, :, :n] = _plain_rows(cache, s["to_table"][b], n, "k").bfloat16()
        v[b, :, :n] = _plain_rows(cache, s["to_table"][b], n, "v").bfloat16()
    return {"idx": idx, "kept": kept, "mass": mass, "k": k, "v": v}


def _plain_cross(s):
    c, q = s["case"], s["q"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    o = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros(q.shape[:3], dtype=torch.float32, device=DEV)
    for b, (L, rows) in enumerate(zip(s["lens_list"], s["rows_list"])):
        if L == 0:
            lse[b, :, :rows] = -math.inf
            continue
        k = s["k"][b, :, :L].float().transpose(1, 2).contiguous()
        v = s["v"][b, :, :L].float()
        step = max(1, 2 ** 28 // (Hq * L))
        for a in range(0, rows, step):
            z = min(rows, a + step)
            x = torch.bmm(q[b, :, a:z].float().reshape(Hkv, -1, D), k) * (1.0 / math.sqrt(D))
            if c["mask"]:
                x.masked_fill_(~s["mask"][b, :L], -math.inf)
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
            l = e.sum(-1, keepdim=True)
            y = torch.bmm(e, v) / torch.where(l == 0, torch.ones_like(l), l)
            o[b, :, a:z] = y.view(Hq, z - a, D).bfloat16()
            lse[b, :, a:z] = (top + torch.log(l)).view(Hq, z - a)
    return {"o": o, "lse": lse}


def _run_plain(s):
    return {"rope": _plain_rope, "mass": _plain_mass, "evict": _plain_evict,
            "cross": _plain_cross}[s["case"]["kind"]](s)


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


def _rope64(case, s):
    """Each pair as a complex number times m e^(i position frequency)."""
    half, N = case["rot"] // 2, case["N"]
    sections = _sections(case)
    m = 1.0
    out = {n: s[n].double().contiguous() for n in ("q", "k")}
    pair = 0
    for axis, size in enumerate(sections):
        for i in range(size):
            index, length = (i, size) if _own_ladders(case) else (pair, half)
            theta = 1.0 / LADDER ** (index / length)
            if case["scaling"] == "ntk" and length > 1:
                theta = 1.0 / (LADDER * FACTOR ** (2.0 * length / (2 * length - 2))) ** (index / length)
            elif case["scaling"] == "linear":
                theta /= FACTOR
            elif case["scaling"] == "parts":
                ends = [length * math.log(CONTEXT / (2 * math.pi * t)) / math.log(LADDER)
                        for t in (32.0, 1.0)]
                first = min(max(math.floor(ends[0]), 0), length - 1)
                last = min(max(math.ceil(ends[1]), 0), length - 1)
                share = min(max((index - first) / max(last - first, 0.001), 0.0), 1.0)
                theta = share * theta / FACTOR + (1.0 - share) * theta
                m = 1.0 + 0.1 * math.log(FACTOR)
            for b in range(case["B"]):
                if "pos" in s:
                    p = s["pos"][axis, b].double()
                else:
                    first_at = int(s["lens"][b] - s["n_new"][b]) if "lens" in s else s["start"]
                    p = torch.arange(first_at, first_at + N, device=DEV, dtype=torch.float64)
                w = torch.polar(torch.full_like(p, m), p * (-theta if case["transpose"] else theta))
                at = (pair, pair + half) if case["layout"] == "half" else (2 * pair, 2 * pair + 1)
                for x in out.values():
                    y = torch.complex(x[b, :, :, at[0]], x[b, :, :, at[1]]) * w
                    x[b, :, :, at[0]], x[b, :, :, at[1]] = y.real, y.imag
            pair += 1
    if "new_list" in s:
        for x in out.values():
            for b, n in enumerate(s["new_list"]):
                x[b, :, n:] = 0.0
    return out


def exact(case, seed):
    s, kv = _inputs(case, seed)
    if case["kind"] == "rope":
        return _rope64(case, s)
    lens, B, D, Hkv = s["lens_list"], case["B"], case["D"], case["Hkv"]
    if case["kind"] == "mass":
        out = torch.zeros(s["mass"].shape, dtype=torch.float64, device=DEV)
        n, share = case["n"], case["Hq"] // Hkv
        for b, L in enumerate(lens):
            out[b, :, :L - n] = s["mass"][b, :, :L - n].double()
            k = _held64(kv(b)[0][0], case["bits"])
            hidden = torch.ones(n, L, dtype=torch.bool, device=DEV).triu(L - n + 1)
            for h in range(case["Hq"]):
                x = s["q"][b, h].double() @ k[h // share].t().contiguous() / math.sqrt(D)
                x -= s["lse"][b, h].double()[:, None]
                x[hidden] = -math.inf
                out[b, h // share, :L] += x.exp().sum(0)
        return {"mass": out}
    if case["kind"] == "evict":
        budget = case["budget"]
        z = dict(dtype=torch.float64, device=DEV)
        mass, k, v = (torch.zeros(B, Hkv, budget, **z), torch.zeros(B, Hkv, budget, D, **z),
                      torch.zeros(B, Hkv, budget, D, **z))
        for b, L in enumerate(lens):
            kb, vb = (_held64(x[0], case["bits"]) for x in kv(b))
            for h in range(Hkv):
                m = s["mass"][b, h, :L].double()
                held = torch.zeros(L, dtype=torch.bool, device=DEV)
                held[:case["sinks"]] = True
                if case["recent"]:
                    held[max(0, L - case["recent"]):] = True
                left = min(budget, L) - int(held.sum())
                if left > 0:
                    rest = torch.nonzero(~held).flatten()
                    order = torch.argsort(-m[rest], stable=True)
                    held[rest[order[:left]]] = True
                at = torch.nonzero(held).flatten()
                mass[b, h, :len(at)] = m[at]
                k[b, h, :len(at)], v[b, h, :len(at)] = kb[h][at], vb[h][at]
        return {"idx": None, "kept": None, "mass": mass, "k": k, "v": v}
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device=DEV)
    share = case["Hq"] // Hkv
    for b, (L, rows) in enumerate(zip(lens, s["rows_list"])):
        at = torch.arange(L, device=DEV)
        if case["mask"]:
            at = at[s["mask"][b, :L]]
        if len(at) == 0:
            lse[b, :, :rows] = -math.inf
            continue
        for h in range(case["Hq"]):
            kh, vh = s["k"][b, h // share][at].double(), s["v"][b, h // share][at].double()
            for r in range(0, rows, 8192):
                x = s["q"][b, h, r:min(rows, r + 8192)].double() @ kh.t().contiguous()
                x /= math.sqrt(D)
                lse[b, h, r:r + len(x)] = x.logsumexp(1)
                o[b, h, r:r + len(x)] = x.softmax(1) @ vh
    return {"o": o, "lse": lse}
