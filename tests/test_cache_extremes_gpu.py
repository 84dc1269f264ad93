"""Window attention, the cache and attention over it at the ends of what they take: magnitudes near
2^100, rows of q that are not finite, memory past 4 GiB, layouts with shared or interleaved rows."""
import math

import pytest
import torch

import paper_2603_29494_amd as va
import sum_bounds as sb
import window_reference as ref

pytestmark = pytest.mark.gpu

ROWS = [(1, 2), (3, 4), (10, 2), (20, 2), (90, 2)]   # 2, 12, 20, 40 and 180 per key/value head


def cached(k, v, bits, page=64):
    """One sequence's cache, its table and length."""
    L, D = k.shape[2:]
    pages = -(-L // page)
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    cache = va.cache_alloc(pages, k.shape[1], D, page, bits)
    cache.data.fill_(0xFF)
    va.cache_write(cache, k, v, table, lens)
    return cache, table, lens


def rows(seed, *shape):
    return sb.rows(seed, *shape).cuda()


def near(o, lse, want):
    assert sb.misses(lse, want[0], want[1]) <= 1 and sb.misses(o, want[2], want[3]) <= 1


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,Hq", ROWS)
@pytest.mark.parametrize("size_k,size_v", [(2.0 ** 97, 1.0), (2.0 ** -90, 1.0), (1.0, 2.0 ** 97),
                                           (1.0, 2.0 ** -90), (2.0 ** 97, 2.0 ** 97)])
def test_magnitudes_of_the_cache(gpu, size_k, size_v, n, Hq, D, bits):
    L = 1300
    k, v = rows(1, 1, 1, L, D) * size_k, rows(2, 1, 1, L, D) * size_v
    q = rows(3, 1, Hq, n, D) / size_k
    cache, table, lens = cached(k, v, bits)
    o, lse = va.cache_attn(q, cache, table, lens, return_lse=True)
    near(o, lse, sb.cache_attn(q, [k[0].cpu()], [v[0].cpu()], bits, [L]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size_k,size_v", [(2.0 ** 97, 1.0), (2.0 ** -90, 1.0), (1.0, 2.0 ** 97),
                                           (1.0, 2.0 ** -90)])
def test_magnitudes_of_the_window(gpu, size_k, size_v, D):
    q, k, v = rows(1, 1, 2, 400, D) / size_k, rows(2, 1, 1, 400, D) * size_k, rows(3, 1, 1, 400, D)
    v = v * size_v
    o, lse = va.window_attn(q, k, v, 150, 5, True, return_lse=True)
    near(o, lse, sb.window_attn(q, k, v, 150, 5, True))


@pytest.mark.parametrize("D,bits", [(64, 8), (128, 4)])
@pytest.mark.parametrize("n,Hq", ROWS[1:])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_a_bad_row_of_q_is_alone(gpu, what, n, Hq, D, bits):
    L = 500
    k, v, q = rows(1, 1, 1, L, D), rows(2, 1, 1, L, D), rows(3, 1, Hq, n, D)
    cache, table, lens = cached(k, v, bits)
    clean = va.cache_attn(q, cache, table, lens, window=200, sinks=3)
    q[0, 1, n // 2, 7] = what
    o = va.cache_attn(q, cache, table, lens, window=200, sinks=3)
    other = torch.ones(1, Hq, n, dtype=torch.bool, device="cuda")
    other[0, 1, n // 2] = False
    assert torch.equal(o[other], clean[other]) and not o[~other].isfinite().any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_a_bad_row_of_q_is_alone_in_a_window(gpu, what, D):
    q, k, v = rows(1, 1, 2, 300, D), rows(2, 1, 1, 300, D), rows(3, 1, 1, 300, D)
    clean = va.window_attn(q, k, v, 100, 3, True)
    q[0, 1, 140, 7] = what
    o = va.window_attn(q, k, v, 100, 3, True)
    other = torch.ones(1, 2, 300, dtype=torch.bool, device="cuda")
    other[0, 1, 140] = False
    assert torch.equal(o[other], clean[other]) and not o[~other].isfinite().any()


@pytest.mark.parametrize("n", [1, 6, 30])   # 4, 24 and 120 rows per key/value head
def test_a_cache_past_4_gib(gpu, n):
    """Pages at both ends of a cache of 5.8 GB, of which nothing else is written."""
    H, D, L, page, pages = 8, 128, 2500, 1024, 2600
    cache = va.cache_alloc(pages, H, D, page, 8)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    k, v, q = rows(1, 1, H, L, D), rows(2, 1, H, L, D), rows(3, 1, 4 * H, n, D)
    va.cache_write(cache, k, v, table, lens)
    gk, gv = va.cache_read(cache, table, lens, L)
    for x, y in ((k, gk), (v, gv)):
        assert torch.equal(y[0].cpu(), torch.stack([ref.held(h.cpu(), 8) for h in x[0]]).bfloat16())
    o, lse = va.cache_attn(q, cache, table, lens, return_lse=True)
    near(o, lse, sb.cache_attn(q, [k[0].cpu()], [v[0].cpu()], 8, [L]))


def test_heads_and_sequences_that_share_rows(gpu):
    """K and V expanded over sequences and heads are written as if copied; rows come back into
    token-major memory between other columns."""
    B, H, n, D = 3, 4, 70, 128
    k, v = rows(1, 1, 1, n, D).expand(B, H, n, D), rows(2, B, 1, n, D).expand(B, H, n, D)
    table = torch.arange(9, dtype=torch.int32, device="cuda").view(3, 3)
    lens = torch.tensor([70, 33, 64], dtype=torch.int32, device="cuda")
    a, b = (va.cache_alloc(9, H, D, 32, 4) for _ in "ab")
    for c in (a, b):
        c.data.zero_()
    va.cache_write(a, k, v, table, lens, n_new=lens)
    va.cache_write(b, k.contiguous(), v.contiguous(), table, lens, n_new=lens)
    assert torch.equal(a.data, b.data)
    buf = torch.full((B, n, 2 * H + 1, D), 3.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    va.cache_read(a, table, lens, n, out=(buf[:, :H], buf[:, H + 1:]))
    gk, gv = va.cache_read(a, table, lens, n)
    for i, L in enumerate(lens.tolist()):
        assert torch.equal(buf[i, :H, :L], gk[i, :, :L])
        assert torch.equal(buf[i, H + 1:, :L], gv[i, :, :L])
        assert (buf[i, :, L:] == 3.0).all()
    assert (buf[:, H] == 3.0).all()


def test_two_graphs_with_one_workspace(gpu):
    """Captured calls of other shapes, replayed in turn, share a workspace and leave each other
    alone."""
    L, D = 5000, 128
    k, v = rows(1, 1, 2, L, D), rows(2, 1, 2, L, D)
    cache, table, lens = cached(k, v, 4)
    qs = [rows(3, 1, 8, 1, D), rows(4, 1, 8, 3, D), rows(5, 1, 8, 60, D)]
    need = [va.cache_attn_workspace_bytes(q, cache, table.shape[1]) for q in qs]
    assert min(need) > 0
    ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.zeros_like(q) for q in qs], []
    for q, out in zip(qs, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            va.cache_attn(q, cache, table, lens, out=out, workspace=ws)
    for L2 in (5000, 100, 4321, 2000):
        lens.fill_(L2)
        ws.fill_(0xFF)
        for i in (0, 2, 1, 0):
            outs[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], va.cache_attn(qs[i], cache, table, lens)), (L2, i)


@pytest.mark.parametrize("start", [0, 417])
def test_a_cached_prompt_in_a_window_layer(gpu, start):
    """New queries over the part of a cached prompt that their window holds, read back as bf16."""
    L, n, window, D = 700, 150, 134, 128     # the first query sees from 417 on
    k, v, q = rows(1, 1, 2, L, D), rows(2, 1, 2, L, D), rows(3, 1, 6, n, D)
    cache, table, lens = cached(k, v, 8)
    gk, gv = va.cache_read(cache, table, lens, L - start, start=start)
    o, lse = va.window_attn(q, gk, gv, window, 0, True, return_lse=True)
    hk, hv = (torch.stack([ref.held(h.cpu(), 8) for h in x[0]])[None].bfloat16() for x in (k, v))
    assert torch.equal(gk.cpu(), hk[:, :, start:]) and torch.equal(gv.cpu(), hv[:, :, start:])
    near(o, lse, sb.window_attn(q, hk, hv, window, 0, True))
