"""Attention over the cache in calls of many sequences or many rows: each way in which the work is
dealt out (cache_deal says which one a case takes), against 64 bits."""
import pytest
import torch

import cache_deal
import paper_2603_29494_amd as va
import sum_bounds as sb

pytestmark = pytest.mark.gpu

PAGE = 64
FORMATS = [(64, 4), (64, 8), (128, 4), (128, 8)]


def spread_lens(B, lo, hi):
    """Lengths all over [lo, hi], in no order."""
    return [lo + (i * 7919 + 13) % B * (hi - lo) // max(1, B - 1) for i in range(B)]


def run(lens, Hq, H, n, D, bits, want, window=None, sinks=0):
    """The call against 64 bits; want(deal, chunk, second, counts) says which case it is."""
    cols = -(-max(lens) // PAGE)
    d = cache_deal.deal(len(lens), Hq, H, n, D, cols, PAGE, window or 1 << 30, sinks)
    seen = cache_deal.blocks_seen(d, lens, n, Hq // H, cols, PAGE, window or 1 << 30, sinks)
    if d.merge:
        chunk, second, counts = cache_deal.chunks(d, H, seen)
        assert sum(counts) * H <= d.items
    else:
        chunk, second, counts = max(seen), False, [1] * len(seen)
    assert want(d, chunk, second, counts), (d, chunk, second)
    per = [-(-L // PAGE) for L in lens]
    ids = torch.randperm(sum(per), generator=torch.Generator().manual_seed(1)).int()
    table = torch.full((len(lens), cols), -1, dtype=torch.int32)
    for b, at in enumerate(torch.tensor([0] + per).cumsum(0)[:-1].tolist()):
        table[b, :per[b]] = ids[at:at + per[b]]
    table, t = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = va.cache_alloc(sum(per), H, D, PAGE, bits)
    cache.data.fill_(0xFF)
    g = torch.Generator(device="cuda").manual_seed(2)
    ks, vs = [], []
    for b, L in enumerate(lens):
        k, v = (torch.randn(1, H, L, D, generator=g, device="cuda").bfloat16() for _ in "kv")
        va.cache_write(cache, k, v, table[b:b + 1], t[b:b + 1])
        ks.append(k[0].cpu())
        vs.append(v[0].cpu())
    q = sb.rows(3, len(lens), Hq, n, D)
    assert va.cache_attn_workspace_bytes(q, cache, cols, window, sinks) == d.workspace
    o, lse = va.cache_attn(q.cuda(), cache, table, t, window=window, sinks=sinks, return_lse=True)
    again = va.cache_attn(q.cuda(), cache, table, t, window=window, sinks=sinks)
    exact = sb.cache_attn(q, ks, vs, bits, lens, window or 1 << 30, sinks)
    assert sb.misses(lse, exact[0], exact[1]) <= 1 and sb.misses(o, exact[2], exact[3]) <= 1
    assert torch.equal(o, again)


@pytest.mark.parametrize("D,bits", FORMATS)
def test_eight_rows_on_four_waves(gpu, D, bits):
    """150 sequences x 2 heads, a few of them long: shares past the first 64 row tiles, two
    workgroups after each other, and a wave per row in the join."""
    lens = spread_lens(146, 1, 300) + [2100, 3000, 2500, 4000]
    run(lens, 16, 2, 1, D, bits, lambda d, chunk, second, counts:
        d.half and d.waves == 4 and d.merge and d.units > 128 and d.target == 1024
        and max(counts[128:]) > 1 and len(lens) * 16 > 2048)


@pytest.mark.parametrize("D,bits", FORMATS[::3])
def test_a_second_chunk_size(gpu, D, bits):
    """Unequal lengths whose last chunks make more of them than there may be."""
    run(spread_lens(60, 1, 5200), 12, 3, 1, D, bits, lambda d, chunk, second, counts:
        d.half and d.waves == 4 and d.merge and second and chunk > d.least)


@pytest.mark.parametrize("D,bits", FORMATS)
def test_more_row_tiles_than_are_dealt_out(gpu, D, bits):
    """One chunk per row tile, one of them of 50 blocks."""
    run(spread_lens(259, 1, 90) + [1590], 4, 1, 1, D, bits, lambda d, chunk, second, counts:
        d.half and d.waves == 4 and not d.merge and d.units == 260 and chunk > d.least)


@pytest.mark.parametrize("D,bits", FORMATS)
@pytest.mark.parametrize("n,Hq", [(1, 16), (2, 14), (1, 40), (20, 8)])
def test_many_sequences_of_more_rows(gpu, n, Hq, D, bits):
    """16, 28, 40 and 160 rows: the other kernels, over 70 sequences."""
    lens = spread_lens(66, n, 300) + [2100, 3000, 2500, 1200]
    run(lens, Hq, 1, n, D, bits, lambda d, chunk, second, counts:
        d.merge and d.units == 70 and max(counts[64:]) > 1 and d.many == (n * Hq > 32)
        and d.waves == (8 if n * Hq > 128 else 4))


@pytest.mark.parametrize("D,bits", FORMATS)
def test_several_row_tiles_of_many_sequences(gpu, D, bits):
    """640 rows of 30 sequences, three row tiles each, with a window and sinks."""
    run(spread_lens(27, 80, 900) + [2600, 1900, 3000], 8, 1, 80, D, bits,
        lambda d, chunk, second, counts: d.many and d.waves == 8 and d.merge and d.units == 90
        and max(counts[64:]) > 1, 1200, 40)
