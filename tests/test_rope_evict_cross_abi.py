"""Refusals of rotary positions, of eviction from the cache and of cross attention, and the host's
ladders of frequencies: no call below reaches the GPU."""
import ctypes
import math

import pytest
import torch

import paper_2603_29494_amd as va
from paper_2603_29494_amd import _lib

OK, INVALID, UNSUPPORTED, CAPACITY = 0, 1, 2, 3
FAKE = 0x100000   # 16-byte aligned address that validation rejects before any use
REF = ctypes.byref


def desc(B, H, N, D, sN=None):
    sN = D if sN is None else sN
    return _lib.TDesc(B, H, N, D, H * N * sN, N * sN, sN)


def cache(data=FAKE, pages=8, H=2, D=128, page=64, bits=4):
    return _lib.CacheDesc(data, pages, H, D, page, bits)


def spec(rot=8, layout=0, axes=1, flags=0, factor=1.0, freq=None, axis=None):
    n = max(1, rot // 2)
    f = (ctypes.c_double * n)(*(freq or [1.0] * n))
    a = None if axis is None else (ctypes.c_int32 * n)(*axis)
    s = _lib.RopeSpec(rot, layout, axes, flags, factor, f, a)
    s.keep = (f, a)
    return s


def test_rope_rejects_bad_arguments():
    lib = _lib.load()

    def rope(q=FAKE, k=FAKE, qo=FAKE + 64, ko=FAKE + 128, qd=None, kd=None, qod=None, kod=None,
             s=None, pos=None, sA=0, sB=0, lens=None, start=1 << 40):
        # that start is refused as well, so that nothing is launched when all else is right
        qd, kd = qd or desc(1, 4, 8, 128), kd or desc(1, 2, 8, 128)
        return lib.vecattn_rope(q, REF(qd), k, REF(kd), REF(s or spec()), pos, sA, sB, lens, None,
                                start, qo, REF(qod or qd), ko, REF(kod or kd), None)
    assert rope() == INVALID                                         # the start
    for name in ("q", "k", "qo", "ko"):
        assert rope(start=0, **{name: None}) == INVALID, name
        assert rope(start=0, **{name: FAKE + 8}) == INVALID, name
    assert rope(start=0, qod=desc(1, 4, 9, 128)) == INVALID
    assert rope(start=0, kod=desc(1, 3, 8, 128)) == INVALID
    assert rope(start=0, kd=desc(1, 2, 9, 128)) == INVALID
    assert rope(start=0, kd=desc(2, 2, 8, 128)) == INVALID
    assert rope(start=0, kd=desc(1, 2, 8, 64)) == INVALID
    # in place with other strides
    assert rope(start=0, qo=FAKE, qod=desc(1, 4, 8, 128, sN=256)) == INVALID
    assert rope(start=0, ko=FAKE, kod=desc(1, 2, 8, 128, sN=256)) == INVALID
    # outputs whose sequences or heads lie on each other, in place or not
    for z in (_lib.TDesc(2, 4, 8, 128, 0, 1024, 128), _lib.TDesc(2, 4, 8, 128, 4096, 0, 128)):
        two = desc(2, 2, 8, 128)
        assert rope(start=0, qd=z, qod=z, kd=two) == INVALID
        assert rope(start=0, qd=z, qo=FAKE, qod=z, kd=two) == INVALID
        assert rope(start=0, qd=desc(2, 4, 8, 128), kd=z, kod=z) == INVALID
    assert rope(start=0, pos=FAKE, lens=FAKE) == INVALID
    assert rope(start=0, pos=FAKE, sA=-1) == INVALID and rope(start=0, pos=FAKE, sB=-1) == INVALID
    assert rope(start=-(1 << 30) - 1) == INVALID and rope(start=(1 << 30) + 1) == INVALID
    for bad in (dict(rot=0), dict(rot=7), dict(rot=130), dict(layout=2), dict(layout=-1),
                dict(axes=0), dict(axes=5), dict(flags=2), dict(flags=4), dict(factor=math.inf),
                dict(factor=math.nan), dict(freq=[1.0, math.nan, 1.0, 1.0]),
                dict(freq=[1.0, 1.0, 1.0, 1025.0]), dict(axis=[0, 0, 0, 1]),
                dict(axis=[0, -1, 0, 0])):
        assert rope(start=0, s=spec(**bad)) == INVALID, bad
    no_freq = spec()
    no_freq.freq = None
    assert rope(start=0, s=no_freq) == INVALID
    assert rope(start=0, qd=desc(1, 4, 8, 64), kd=desc(1, 2, 8, 64), s=spec(rot=66)) == INVALID
    assert rope(start=0, qd=desc(1, 4, 8, 96)) == UNSUPPORTED
    assert rope(start=0, qd=desc(1, 65535, 8, 64), kd=desc(1, 1, 8, 64)) == UNSUPPORTED
    many = 1 << 26
    assert rope(start=0, qd=desc(many, 1, 17, 64), kd=desc(many, 1, 17, 64)) == UNSUPPORTED


def test_ladders():
    f, m = va.rope_ladder(16)
    assert m == 1.0 and len(f) == 8
    for i in range(8):
        assert f[i] == pytest.approx(10000.0 ** (-2 * i / 16), rel=1e-15)
    lin, _ = va.rope_ladder(16, scaling="linear", factor=4.0)
    assert lin == pytest.approx([x / 4 for x in f], rel=1e-15)
    ntk, m = va.rope_ladder(16, scaling="ntk", factor=4.0)
    assert m == 1.0 and ntk[0] == f[0] and ntk[7] == pytest.approx(f[7] / 4, rel=1e-14)
    assert all(a <= b for a, b in zip(ntk, f))
    parts, m = va.rope_ladder(128, scaling="parts", factor=16.0, context=8192)
    full, _ = va.rope_ladder(128)
    assert m == pytest.approx(1 + 0.1 * math.log(16.0))
    turns = [8192 * x / (2 * math.pi) for x in full]
    for x, y, t in zip(parts, full, turns):
        if t >= 32 * full[0] / full[1]:          # a step above the border: kept
            assert x == y
        elif t <= full[1] / full[0]:             # a step below: divided
            assert x == pytest.approx(y / 16, rel=1e-15)
        else:
            assert y / 16 <= x <= y
    share = [x / y for x, y in zip(parts, full)]
    steps = [a - b for a, b in zip(share, share[1:])]
    some = [s for s in steps if s > 1e-9]
    assert max(some) - min(some) < 1e-9          # linear in the pair
    bands, m = va.rope_ladder(128, scaling="bands", factor=8.0, context=8192, fast=4.0, slow=1.0)
    assert m == 1.0
    for x, y, t in zip(bands, full, turns):
        s = min(max((t - 1.0) / 3.0, 0.0), 1.0)
        assert x == pytest.approx(s * y + (1 - s) * y / 8, rel=1e-13)
    assert va.rope_ladder(2, scaling="ntk", factor=3.0)[0] == (1.0,)
    for scaling in (None, "linear", "ntk", "parts", "bands"):   # one pair, nothing stretched
        assert va.rope_ladder(2, scaling=scaling, factor=1.0, context=100)[0] == (1.0,)
    for bad in (dict(rot=3), dict(rot=0), dict(rot=130), dict(base=1.0), dict(base=math.inf),
                dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=math.nan),
                dict(scaling="parts", context=0), dict(scaling="parts", context=9, slow=0.0),
                dict(scaling="bands", context=9, fast=1.0, slow=1.0),
                dict(scaling="bands", context=math.inf)):
        with pytest.raises(va.VecattnError) as e:
            va.rope_ladder(**dict(dict(rot=16), **bad))
        assert e.value.status == INVALID, bad
    with pytest.raises(ValueError):
        va.rope_ladder(16, scaling="cubic")
    lib, m = _lib.load(), ctypes.c_double()
    assert lib.vecattn_rope_ladder(16, 1e4, 5, 1.0, 1.0, 2.0, 1.0, FAKE, REF(m)) == INVALID
    assert lib.vecattn_rope_ladder(16, 1e4, 0, 1.0, 1.0, 2.0, 1.0, None, REF(m)) == INVALID


def test_plans():
    p = va.rope_plan(24, sections=(2, 5, 5))
    assert p.axes == 3 and p.axis == (0,) * 2 + (1,) * 5 + (2,) * 5
    assert p.freq == va.rope_ladder(24)[0]
    own = va.rope_plan(24, sections=(2, 5, 5), own_ladders=True)
    assert own.freq == va.rope_ladder(4)[0] + 2 * va.rope_ladder(10)[0]
    for bad in (dict(sections=(2, 5)), dict(sections=(12, 0)), dict(layout="both"), dict(rot=25)):
        with pytest.raises(ValueError):
            va.rope_plan(**dict(dict(rot=24), **bad))


def test_cache_mass_rejects_bad_arguments():
    lib = _lib.load()

    def mass(q=FAKE, qd=None, lse=FAKE, c=None, table=FAKE, cols=4, lens=FAKE, window=8, sinks=0,
             scale=0.0, decay=-1.0, out=FAKE, M=256, flags=0, ws=None,
             nws=0):
        # decay = -1 is refused as well
        return lib.vecattn_cache_mass(q, REF(qd or desc(2, 4, 1, 128)), lse, REF(c or cache()), table,
                                      cols, lens, None, window, sinks, scale, decay, None, out, M,
                                      flags, ws, nws, None)
    assert mass() == INVALID
    for name in ("q", "lse", "table", "lens", "out"):
        assert mass(decay=1.0, **{name: None}) == INVALID, name
    assert mass(decay=math.nan) == INVALID and mass(decay=math.inf) == INVALID
    for bad in (dict(q=FAKE + 8), dict(window=0), dict(sinks=-1), dict(scale=-1.0), dict(M=0),
                dict(scale=math.nan), dict(M=(1 << 30) + 1), dict(cols=0), dict(c=cache(data=None)),
                dict(flags=1),
                dict(c=cache(D=64)), dict(qd=desc(2, 3, 1, 128)), dict(c=cache(bits=2))):
        assert mass(decay=1.0, **bad) == INVALID, bad
    assert mass(decay=1.0, qd=desc(2, 4, 1, 80)) == UNSUPPORTED
    assert mass(decay=1.0, qd=desc(1, 4, 1 << 28, 128)) == UNSUPPORTED
    # more than 48 rows need a workspace
    n, many = ctypes.c_size_t(9), desc(2, 4, 25, 128)
    assert lib.vecattn_cache_mass_workspace_size(REF(desc(2, 4, 24, 128)), REF(cache()), REF(n)) == OK
    assert n.value == 0
    assert lib.vecattn_cache_mass_workspace_size(REF(many), REF(cache()), REF(n)) == OK
    assert n.value > 0
    assert mass(decay=1.0, qd=many) == CAPACITY
    assert mass(decay=1.0, qd=many, ws=FAKE, nws=n.value - 1) == CAPACITY
    assert mass(decay=1.0, qd=many, ws=FAKE + 8, nws=n.value) == INVALID
    assert lib.vecattn_cache_mass_workspace_size(REF(many), REF(cache()), None) == INVALID
    assert lib.vecattn_cache_mass_workspace_size(REF(many), REF(cache(H=3)), REF(n)) == INVALID


def test_cache_keep_and_gather_reject_bad_arguments():
    lib = _lib.load()

    def keep(mass=FAKE, M=256, B=2, c=None, table=FAKE, cols=4, lens=FAKE, budget=8, sinks=0,
             recent=9, idx=FAKE, kept=FAKE, ws=None, nws=0):
        # recent = 9 is more than the budget
        return lib.vecattn_cache_keep(mass, M, B, REF(c or cache()), table, cols, lens, budget, sinks,
                                      recent, idx, kept, ws, nws, None)
    assert keep() == INVALID
    for name in ("mass", "table", "lens", "idx", "kept"):
        assert keep(recent=0, **{name: None}) == INVALID, name
    for bad in (dict(M=0), dict(M=(1 << 30) + 1), dict(B=0), dict(budget=0), dict(sinks=-1),
                dict(budget=(1 << 30) + 1), dict(recent=-1), dict(sinks=4, recent=5),
                dict(sinks=1 << 62, recent=1 << 62), dict(cols=0), dict(cols=1 << 25),
                dict(c=cache(page=33)), dict(c=cache(data=None))):
        assert keep(**dict(dict(recent=0), **bad)) == INVALID, bad
    assert keep(recent=0, B=70000) == UNSUPPORTED
    assert keep(recent=0, c=cache(D=96)) == UNSUPPORTED
    # more than 32768 tokens need a workspace
    n = ctypes.c_size_t(9)
    size = lib.vecattn_cache_keep_workspace_size
    assert size(REF(cache()), 512, 2, 1 << 20, REF(n)) == OK and n.value == 0
    assert size(REF(cache()), 513, 2, 1 << 20, REF(n)) == OK and n.value > 0
    long = dict(recent=0, cols=513, M=1 << 20)
    assert keep(**long) == CAPACITY and keep(ws=FAKE, nws=n.value - 1, **long) == CAPACITY
    assert keep(ws=FAKE + 8, nws=n.value, **long) == INVALID
    assert size(REF(cache()), 0, 2, 64, REF(n)) == INVALID
    assert size(REF(cache()), 4, 0, 64, REF(n)) == INVALID
    assert size(REF(cache()), 4, 2, 0, REF(n)) == INVALID
    assert size(REF(cache()), 4, 2, 64, None) == INVALID
    assert size(REF(cache()), 4, 70000, 64, REF(n)) == UNSUPPORTED

    def gather(c=None, table=FAKE, cols=4, B=2, idx=FAKE, kept=FAKE, budget=8, to=None,
               to_table=FAKE, to_cols=0, mass=FAKE, M=256, mass_out=FAKE, flags=0):
        # to_cols = 0 is refused as well
        return lib.vecattn_cache_gather(REF(c or cache()), table, cols, B, idx, kept, budget,
                                        REF(to or cache()), to_table, to_cols, mass, M, mass_out,
                                        flags, None)
    assert gather() == INVALID
    for name in ("table", "idx", "kept", "to_table", "mass", "mass_out"):
        assert gather(to_cols=4, **{name: None}) == INVALID, name
    for bad in (dict(cols=0), dict(B=0), dict(budget=0), dict(M=0), dict(to=cache(H=3)),
                dict(to=cache(D=64)), dict(to=cache(bits=8)), dict(to=cache(data=None)),
                dict(c=cache(data=FAKE + 4)), dict(to_cols=1 << 25), dict(flags=2)):
        assert gather(**dict(dict(to_cols=4), **bad)) == INVALID, bad
    assert gather(to_cols=4, B=70000) == UNSUPPORTED


def test_cross_attn_rejects_bad_arguments():
    lib = _lib.load()

    def cross(q=FAKE, k=FAKE, v=FAKE, o=FAKE, qd=None, kd=None, vd=None, od=None, mask=None, sB=0,
              scale=-1.0, flags=0, ws=None, nws=0):
        # scale = -1 is refused as well
        qd, kd = qd or desc(1, 4, 64, 128), kd or desc(1, 2, 77, 128)
        return lib.vecattn_cross_attn(q, REF(qd), k, REF(kd), v, REF(vd or kd), None, mask, sB, None,
                                      flags, scale, o, REF(od or qd), None, ws, nws, None)
    assert cross() == INVALID
    for name in "qkvo":
        assert cross(scale=0.0, **{name: None}) == INVALID
        assert cross(scale=0.0, **{name: FAKE + 8}) == INVALID
    for bad in (dict(scale=math.nan), dict(sB=-1), dict(flags=1), dict(qd=desc(1, 3, 64, 128)),
                dict(kd=desc(2, 2, 77, 128)), dict(kd=desc(1, 2, 77, 64)),
                dict(vd=desc(1, 2, 78, 128)), dict(od=desc(1, 4, 63, 128)), dict(ws=FAKE + 8, nws=64)):
        assert cross(**dict(dict(scale=0.0), **bad)) == INVALID, bad
    for z in (_lib.TDesc(2, 4, 64, 128, 0, 8192, 128), _lib.TDesc(2, 4, 64, 128, 32768, 0, 128)):
        assert cross(scale=0.0, qd=desc(2, 4, 64, 128), od=z, kd=desc(2, 2, 77, 128)) == INVALID
    assert cross(scale=0.0, qd=desc(1, 4, 64, 80)) == UNSUPPORTED
    assert cross(scale=0.0, kd=desc(1, 2, 77, 128, sN=1 << 24)) == UNSUPPORTED
    assert cross(scale=0.0, vd=desc(1, 2, 77, 128, sN=1 << 24)) == UNSUPPORTED
    assert cross(scale=0.0, qd=desc(1, 4, 1 << 30, 128)) == UNSUPPORTED       # rows
    assert cross(scale=0.0, qd=desc(1 << 14, 4096, 1, 64), kd=desc(1 << 14, 4096, 1, 64)) == UNSUPPORTED
    # one row over many keys needs a workspace
    n = ctypes.c_size_t(0)
    one, far = desc(1, 4, 1, 128), desc(1, 4, 20000, 128)
    assert lib.vecattn_cross_attn_workspace_size(REF(one), REF(far), REF(n)) == OK and n.value > 0
    assert cross(scale=0.0, qd=one, kd=far) == CAPACITY
    assert cross(scale=0.0, qd=one, kd=far, ws=FAKE, nws=n.value - 1) == CAPACITY
    assert lib.vecattn_cross_attn_workspace_size(REF(one), REF(far), None) == INVALID
    assert lib.vecattn_cross_attn_workspace_size(None, REF(far), REF(n)) == INVALID
    assert lib.vecattn_cross_attn_workspace_size(REF(one), REF(desc(1, 3, 5, 128)), REF(n)) == INVALID


def test_binding_checks_on_the_host():
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    plan = va.rope_plan(64)
    for call in (lambda: va.rope(plan, x), lambda: va.cross_attn(x, x, x)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        va.Rope("half", (1.0,), (0, 1))
    with pytest.raises(ValueError):
        va.Rope("half", (), ())
