"""Eviction at sizes that change how the work is dealt out: waves that walk over several blocks of
tokens, and calls of several launches on several streams at once."""
import pytest
import torch

import paper_2603_29494_amd as va
from test_cache_gpu import fresh_cache, int32, paged, rows
from test_evict_gpu import check_mass, keep_ref, mass64, setup

pytestmark = pytest.mark.gpu

B, H = 16, 8   # 128 heads: 64 waves for each, of up to 256 blocks of 32 tokens


@pytest.mark.parametrize("D,bits,page", [(128, 4, 64), (64, 8, 32)])
@pytest.mark.parametrize("group,n", [(7, 1), (4, 4), (7, 4), (6, 8)])
def test_waves_that_walk_over_blocks(gpu, D, bits, page, group, n):
    """Up to 8, 16, 32 and 48 rows.  A token's sum is of one wave in one order, however many blocks
    that wave has: a sequence alone (a block each) gives the same bits, and two of them are checked
    against 64 bits."""
    lens = [8192 - 531 * b for b in range(B - 1)] + [n]
    n_new = [n] * B
    n_new[3], n_new[4] = 0, 1
    ks, cache, table, q, _ = setup(D, bits, page, lens, H, group, n)
    table[2, 5] = -1                       # pages that are not held, one in the middle of a walk
    table[6, lens[6] // page - 1] = 1 << 28
    M = 8192 + 40
    old = torch.rand(B, H, M, generator=torch.Generator().manual_seed(1)).cuda()
    ld, nd = int32(lens), int32(n_new)
    for window, sinks, decay in ((None, 0, 1.0), (700, 90, 0.5)):
        _, lse = va.cache_attn(q, cache, table, ld, n_new=nd, window=window, sinks=sinks,
                               return_lse=True)
        kw = dict(window=window, sinks=sinks, decay=decay)
        state, apart = old.clone(), torch.full_like(old, -7.0)
        va.cache_mass(q, lse, cache, table, ld, mass=state, n_new=nd, out=state, **kw)
        va.cache_mass(q, lse, cache, table, ld, mass=old, n_new=nd, out=apart, **kw)
        made = va.cache_mass(q, lse, cache, table, ld, mass=old, n_new=nd, **kw)
        torch.cuda.synchronize()
        for b in range(B):
            z = slice(b, b + 1)
            one = va.cache_mass(q[z], lse[z], cache, table[z], ld[z], mass=old[z], n_new=nd[z], **kw)
            L = lens[b]
            for got, past in ((state, old[b, :, L:]), (apart, -7.0), (made, 0.0)):
                assert torch.equal(got[b, :, :L], one[0, :, :L]), b
                assert (got[b, :, L:] == past).all()
        for b in (1, 2):
            hidden = torch.zeros(lens[b], dtype=torch.bool)
            if b == 2:
                hidden[5 * page:6 * page] = True
            refs = mass64(q[b:b + 1], lse[b:b + 1], ks[b:b + 1], bits, lens[b:b + 1], old[b:b + 1],
                          n_new[b:b + 1], window or 1 << 30, sinks, decay=decay, hidden=[hidden])
            check_mass(made[b:b + 1], refs, 0.0)


def test_calls_of_several_launches_at_once(gpu):
    """Rows prepared, split and joined, and long rows kept over six launches: each call has a
    workspace of its own, and gives what it gives alone."""
    ks, cache, table, q, lse = setup(64, 4, 32, [700, 300], 2, 4, 160)
    lens = int32([700, 300])
    M, page = 70000, 64
    cols = -(-M // page)
    long = fresh_cache(2 * cols, 2, 64, page, 4)
    pages = torch.randperm(2 * cols, generator=torch.Generator().manual_seed(2)).int().view(2, -1).cuda()
    held = int32([M, 40001])
    g = torch.Generator().manual_seed(3)
    masses = [torch.exp(3 * torch.randn(2, 2, M, generator=g)).cuda() for _ in range(3)]
    qs = [q, rows(31, *q.shape), rows(32, *q.shape)]
    assert va.cache_mass_workspace_bytes(q, cache) > 0
    assert va.cache_keep_workspace_bytes(masses[0], long, cols) > 0

    def call(i):
        return (va.cache_mass(qs[i], lse, cache, table, lens),
                *va.cache_keep(masses[i], long, pages, held, 9000, 16, 100))
    alone = [call(i) for i in range(3)]
    torch.cuda.synchronize()
    for i, (_, idx, kept) in enumerate(alone):
        assert kept.tolist() == [9000, 9000]
        for b, L in enumerate((M, 40001)):
            assert idx[b, 1].tolist() == keep_ref(masses[i][b, 1].tolist(), range(L), L, 9000, 16, 100)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(3):
        outs = []
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append(call(i))
        torch.cuda.synchronize()
        for a, b in zip(outs, alone):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_gather_and_read_back_at_once(gpu):
    """Several streams cut the same cache into pages of their own."""
    lens, budget = [3000, 900], 700
    k = rows(1, 2, 2, 3000, 128)
    table, pages = paged(lens, 64)
    to, more = paged([budget, budget], 64, 5)
    cache = fresh_cache(pages + 3 * more, 2, 128, 64, 4)
    va.cache_write(cache, k, k, table, int32(lens), n_new=int32(lens))
    mass = torch.rand(2, 2, table.shape[1] * 64, generator=torch.Generator().manual_seed(6)).cuda()
    idx, kept = va.cache_keep(mass, cache, table, int32(lens), budget, 4, 60)
    sk, sv = va.cache_read(cache, table, int32(lens), 3000)
    tables = [torch.where(to >= 0, to + pages + i * more, to) for i in range(3)]
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream() for _ in range(3)]
    for s, t in zip(streams, tables):
        with torch.cuda.stream(s):
            left = va.cache_gather(cache, table, idx, kept, t, mass=mass)
            outs.append((left, *va.cache_read(cache, t, kept, budget)))
    torch.cuda.synchronize()
    at = idx.long()
    for left, gk, gv in outs:
        assert torch.equal(left, mass.gather(2, at))
        for got, src in ((gk, sk), (gv, sv)):
            assert torch.equal(got, src.gather(2, at[..., None].expand(-1, -1, -1, 128)))
