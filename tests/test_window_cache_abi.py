"""Refusals of the window attention and of the quantised cache's entry points, on the host: every
call below fails validation before any launch."""
import ctypes

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


def test_window_attn_rejects_bad_arguments():
    lib = _lib.load()

    def win(q=FAKE, k=FAKE, v=FAKE, o=FAKE, qd=None, kd=None, vd=None, od=None, window=8, sinks=0,
            causal=0, scale=-1.0):
        # scale = -1 is refused as well, so that nothing is launched when all else is right
        qd, kd = qd or desc(1, 4, 64, 128), kd or desc(1, 2, 128, 128)
        vd, od = vd or desc(1, 2, 128, 128), od or desc(1, 4, 64, 128)
        return lib.vecattn_window_attn(q, REF(qd), k, REF(kd), v, REF(vd), None, window, sinks,
                                       causal, scale, o, REF(od), None, None)
    assert win() == INVALID                                            # the scale
    for name in "qkvo":
        assert win(**{name: None}) == INVALID
        assert win(**{name: FAKE + 8}) == INVALID
    assert win(scale=0.0, window=0) == INVALID and win(scale=0.0, sinks=-1) == INVALID
    assert win(scale=0.0, causal=2) == INVALID and win(scale=float("nan")) == INVALID
    assert win(scale=0.0, qd=desc(1, 4, 129, 128), od=desc(1, 4, 129, 128)) == INVALID  # Nq > Nk
    assert win(scale=0.0, qd=desc(1, 3, 64, 128), od=desc(1, 3, 64, 128)) == INVALID
    assert win(scale=0.0, vd=desc(1, 2, 127, 128)) == INVALID
    assert win(scale=0.0, od=desc(1, 4, 63, 128)) == INVALID
    assert win(scale=0.0, kd=desc(1, 2, 128, 64)) == INVALID
    assert win(scale=0.0, qd=desc(1, 4, 64, 96)) == UNSUPPORTED
    big = 70000
    assert win(scale=0.0, qd=desc(big, 2, 8, 64), kd=desc(big, 2, 8, 64), vd=desc(big, 2, 8, 64),
               od=desc(big, 2, 8, 64)) == UNSUPPORTED
    many = desc(60000, 64, 300, 64)
    assert win(scale=0.0, qd=many, kd=many, vd=many, od=many) == UNSUPPORTED
    wide = desc(1, 2, 128, 128, sN=1 << 24)
    assert win(scale=0.0, kd=wide) == UNSUPPORTED and win(scale=0.0, vd=wide) == UNSUPPORTED


def test_cache_size():
    # codes and one bf16 pair per 64 values, K and V
    assert va.cache_bytes(10, 4, 128, 64, 4) == 10 * 4 * 64 * 2 * (64 + 8)
    assert va.cache_bytes(3, 1, 64, 32, 8) == 3 * 32 * 2 * (64 + 4)
    for bad in (dict(pages=0), dict(heads=0), dict(page=16), dict(page=48), dict(page=2048),
                dict(bits=3), dict(dim=0), dict(pages=1 << 62)):
        args = dict(dict(pages=2, heads=2, dim=128), **bad)
        with pytest.raises(va.VecattnError) as e:
            va.cache_bytes(**args)
        assert e.value.status == INVALID, bad
    for bad in (dict(dim=96), dict(heads=70000)):
        with pytest.raises(va.VecattnError) as e:
            va.cache_bytes(**dict(dict(pages=2, heads=2, dim=128), **bad))
        assert e.value.status == UNSUPPORTED
    assert _lib.load().vecattn_cache_size(None, None) == INVALID


def test_cache_write_and_read_reject_bad_arguments():
    lib = _lib.load()

    def write(k=FAKE, v=FAKE, kd=None, vd=None, c=None, table=FAKE, cols=4, lens=FAKE):
        kd = kd or desc(1, 2, 8, 128)
        vd = vd or kd
        return lib.vecattn_cache_write(k, REF(kd), v, REF(vd), REF(c or cache()), table, cols, lens,
                                       None, None)

    def read(k=FAKE, v=FAKE, kd=None, vd=None, c=None, table=FAKE, cols=4, lens=FAKE, start=0):
        kd = kd or desc(1, 2, 8, 128)
        vd = vd or kd
        return lib.vecattn_cache_read(REF(c or cache()), table, cols, lens, start, k, REF(kd), v,
                                      REF(vd), None)
    for call in (write, read):
        for name in ("k", "v", "table", "lens"):
            assert call(**{name: None}) == INVALID, name
        assert call(k=FAKE + 4) == INVALID and call(v=FAKE + 2) == INVALID
        assert call(cols=0) == INVALID and call(cols=(1 << 24) + 1) == INVALID
        assert call(c=cache(data=None)) == INVALID and call(c=cache(data=FAKE + 8)) == INVALID
        assert call(c=cache(bits=5)) == INVALID and call(c=cache(page=96)) == INVALID
        assert call(c=cache(H=3)) == INVALID and call(c=cache(D=64)) == INVALID
        assert call(vd=desc(1, 2, 9, 128)) == INVALID
        assert call(kd=desc(1, 2, 8, 96)) == UNSUPPORTED
        assert call(kd=desc(1, 2, (1 << 28) + 8, 128)) == UNSUPPORTED
        assert call(kd=desc(70000, 2, 8, 128)) == UNSUPPORTED
    assert read(start=-1) == INVALID and read(start=(1 << 30) + 1) == INVALID


def test_cache_attn_rejects_bad_arguments():
    lib = _lib.load()

    def attn(q=FAKE, o=FAKE, qd=None, od=None, c=None, table=FAKE, cols=4, lens=FAKE, window=8,
             sinks=0, scale=0.0, ws=None, nws=0):
        qd = qd or desc(2, 4, 1, 128)
        od = od or qd
        return lib.vecattn_cache_attn(q, REF(qd), REF(c or cache()), table, cols, lens, None, window,
                                      sinks, scale, o, REF(od), None, ws, nws, None)
    for name in ("q", "o", "table", "lens"):
        assert attn(**{name: None}) == INVALID, name
    assert attn(q=FAKE + 8) == INVALID and attn(window=0) == INVALID and attn(sinks=-1) == INVALID
    assert attn(scale=-1.0) == INVALID and attn(scale=float("inf")) == INVALID
    assert attn(cols=0) == INVALID and attn(c=cache(data=None)) == INVALID
    assert attn(qd=desc(2, 3, 1, 128)) == INVALID and attn(c=cache(D=64)) == INVALID
    assert attn(od=desc(2, 4, 2, 128)) == INVALID
    assert attn(qd=desc(2, 4, 1, 80)) == UNSUPPORTED
    assert attn(qd=desc(1, 4, 1 << 28, 128)) == UNSUPPORTED     # past the launch limits
    # a long table needs a workspace
    n = ctypes.c_size_t(0)
    qd, c = desc(1, 4, 1, 128), cache(pages=4096)
    assert lib.vecattn_cache_attn_workspace_size(REF(qd), REF(c), 2048, 1 << 30, 0,
                                                 REF(n)) == OK and n.value > 0
    big = dict(qd=qd, c=c, cols=2048, window=1 << 30)
    assert attn(**big) == CAPACITY
    assert attn(**big, ws=FAKE, nws=n.value - 1) == CAPACITY
    assert attn(**big, ws=FAKE + 8, nws=n.value) == INVALID
    assert lib.vecattn_cache_attn_workspace_size(REF(qd), REF(c), 2048, 0, 0, REF(n)) == INVALID
    assert lib.vecattn_cache_attn_workspace_size(None, REF(c), 2048, 1, 0, REF(n)) == INVALID
    assert lib.vecattn_cache_attn_workspace_size(REF(qd), REF(c), 2048, 1, 0, None) == INVALID


def test_workspace_follows_what_a_row_can_see():
    q = torch.empty(1, 4, 1, 128, dtype=torch.bfloat16)
    c = va.Cache(torch.empty(va.cache_bytes(4096, 4, 128), dtype=torch.uint8), 4096, 4, 128, 64, 4)
    whole = va.cache_attn_workspace_bytes(q, c, 2048)
    assert whole > va.cache_attn_workspace_bytes(q, c, 2048, window=4096) > 0
    assert va.cache_attn_workspace_bytes(q, c, 2048, window=100) == 0
    assert va.cache_attn_workspace_bytes(q, c, 1) == 0


def test_binding_rejects_what_is_not_on_the_gpu():
    x = torch.zeros(1, 2, 8, 128, dtype=torch.bfloat16)
    c = va.Cache(torch.empty(va.cache_bytes(2, 2, 128), dtype=torch.uint8), 2, 2, 128, 64, 4)
    table, lens = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        va.window_attn(x, x, x, 8)
    with pytest.raises(TypeError):
        va.cache_write(c, x, x, table, lens)
    with pytest.raises(TypeError):
        va.cache_attn(x, c, table, lens)
    with pytest.raises(ValueError):
        va.cache_read(c, table, lens, 4)
    with pytest.raises(ValueError):
        va.Cache(c.data[:-1], 2, 2, 128, 64, 4)     # a byte short


# ---- the 64-bit forms themselves, on small cases ----

def test_reference_format_on_worked_values():
    import window_reference as ref
    x = torch.zeros(1, 64, dtype=torch.bfloat16)
    x[0, :4] = torch.tensor([-1.0, 2.0, 0.1, 14.0])
    u, m, s = ref.quantise(x, 4)
    assert m.item() == -1.0 and s.item() == 1.0
    assert u[0, :5].tolist() == [0, 3, 1, 15, 1]
    x[0, 5] = float("nan")
    assert ref.held(x, 4).isnan().all()


def test_reference_window_is_a_masked_softmax():
    import window_reference as ref
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(1, 1, 9, 64, generator=g).bfloat16() for _ in range(3))
    o, lse, _, _ = ref.window_attn(q, k, v, 2, 1, True)
    s = (q[0, 0].double() @ k[0, 0].double().t()) / 8.0
    for p in range(9):
        seen = sorted({0, max(0, p - 1), p})
        w = torch.softmax(s[p, seen], 0)
        assert torch.allclose(o[0, 0, p], w @ v[0, 0, seen].double(), atol=1e-12)
        assert torch.allclose(lse[0, 0, p], torch.logsumexp(s[p, seen], 0), atol=1e-12)
