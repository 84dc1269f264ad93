"""Caches that are cut, written on behind what was kept, and cut again: new tokens have entries
among the collected weights, also past the first budget."""
import pytest
import torch

import paper_2603_29494_amd as va
from test_cache_gpu import fresh_cache, int32, paged, rows
from test_evict_gpu import check_mass, keep_ref, mass64

pytestmark = pytest.mark.gpu

H, GROUP, PAGE, BUDGET = 2, 2, 32, 64


def cut(D, bits, lens):
    """A cache of these sequences cut to BUDGET: what the second step starts from.  The table has
    pages for 160 slots."""
    table, pages = paged(lens, PAGE)
    cache = fresh_cache(pages + 5 * len(lens), H, D, PAGE, bits)
    for b, L in enumerate(lens):
        k = rows(10 + b, 1, H, L, D)
        va.cache_write(cache, k, k, table[b:b + 1], int32([L]))
    q = rows(5, len(lens), H * GROUP, 1, D)
    _, lse = va.cache_attn(q, cache, table, int32(lens), return_lse=True)
    mass = va.cache_mass(q, lse, cache, table, int32(lens))
    idx, kept = va.cache_keep(mass, cache, table, int32(lens), BUDGET, sinks=4, recent=8)
    to = torch.arange(pages, pages + 5 * len(lens), dtype=torch.int32, device="cuda").view(-1, 5)
    return cache, table, mass, idx, kept, to


def append(cache, to, kept, n, D, seed):
    """n tokens behind the kept ones: their keys, q and lse."""
    B = kept.shape[0]
    k, q = rows(seed, B, H, n, D), rows(seed + 1, B, H * GROUP, n, D)
    held = kept + n
    va.cache_write(cache, k, k, to, held)
    _, lse = va.cache_attn(q, cache, to, held, return_lse=True)
    return k, q, lse, held


@pytest.mark.parametrize("D,bits", [(128, 4), (64, 8)])
@pytest.mark.parametrize("n", [1, 5, 70])
def test_new_tokens_past_the_budget_collect_and_are_kept(gpu, D, bits, n):
    """What cache_gather returns goes into cache_mass as it is: the weights come out with an entry
    for each token of the table, and `recent` ones past the first budget survive the second cut."""
    lens = [300, 64, 90]
    cache, table, mass, idx, kept, to = cut(D, bits, lens)
    left = va.cache_gather(cache, table, idx, kept, to, mass=mass)
    assert kept.tolist() == [BUDGET] * 3
    k, q, lse, held = append(cache, to, kept, n, D, 20)
    got = va.cache_mass(q, lse, cache, to, held, mass=left, decay=0.5)
    assert got.shape == (3, H, 5 * PAGE)
    # the same, in a tensor with room for all
    state = torch.full((3, H, 5 * PAGE), -7.0, device="cuda")
    state[:, :, :BUDGET] = left
    want = va.cache_mass(q, lse, cache, to, held, mass=state, decay=0.5)
    assert torch.equal(got, want) and (got[:, :, BUDGET + n:] == 0).all()
    assert (got[:, :, BUDGET:BUDGET + n] > 0).all()
    budget, recent = 40, 24
    again, count = va.cache_keep(got, cache, to, held, budget, sinks=4, recent=recent)
    assert count.tolist() == [budget] * 3
    for b in range(3):
        L = BUDGET + n
        for h in range(H):
            ref = keep_ref(got[b, h].tolist(), range(L), L, budget, 4, recent)
            assert again[b, h].tolist() == ref
            assert set(range(L - recent, L)) <= set(ref)


@pytest.mark.parametrize("D,bits", [(128, 8), (64, 4)])
def test_room_for_the_tokens_to_come(gpu, D, bits):
    """cache_gather with an entry for each token of the table, in place from there on, the second
    step as a graph that is replayed."""
    lens = [300, 20, 90]
    cache, table, mass, idx, kept, to = cut(D, bits, lens)
    left = va.cache_gather(cache, table, idx, kept, to, mass=mass)
    for entries in (BUDGET, BUDGET + 1, 5 * PAGE, 5000):
        junk = torch.full((3, H, entries), 7.0, device="cuda")
        del junk
        wide = va.cache_gather(cache, table, idx, kept, to, mass=mass, entries=entries)
        assert wide.shape == (3, H, entries)
        assert torch.equal(wide[:, :, :BUDGET], left) and (wide[:, :, BUDGET:] == 0).all()
    state = va.cache_gather(cache, table, idx, kept, to, mass=mass, entries=5 * PAGE)
    k, q, lse, held = append(cache, to, kept, 9, D, 40)
    want = va.cache_mass(q, lse, cache, to, held, mass=left)
    first = state.clone()

    def step():
        va.cache_mass(q, lse, cache, to, held, mass=state, out=state)
        return va.cache_keep(state, cache, to, held, 30, sinks=2, recent=12)
    ref = step()
    assert torch.equal(state, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        state.copy_(first)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(state, want)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    for b in range(3):
        L = int(held[b])
        for h in range(H):
            assert set(range(L - 12, L)) <= set(ref[0][b, h].tolist())


def test_sums_of_padded_weights(gpu):
    """Against 64 bits, from collected weights shorter than the table, with padded rows."""
    lens, n = [100, 700, 3], 4
    n_new = int32([4, 2, 0])
    table, pages = paged(lens, PAGE)
    cache = fresh_cache(pages, H, 64, PAGE, 8)
    ks = [rows(60 + b, H, L, 64) for b, L in enumerate(lens)]
    for b, L in enumerate(lens):
        va.cache_write(cache, ks[b][None], ks[b][None], table[b:b + 1], int32([L]))
    q = rows(70, 3, H * GROUP, n, 64)
    _, lse = va.cache_attn(q, cache, table, int32(lens), n_new=n_new, return_lse=True)
    old = torch.rand(3, H, 50, generator=torch.Generator().manual_seed(1)).cuda()
    keep = old.clone()
    got = va.cache_mass(q, lse, cache, table, int32(lens), mass=old, n_new=n_new, decay=0.25)
    assert got.shape == (3, H, table.shape[1] * PAGE) and torch.equal(old, keep)
    full = torch.cat([old.cpu(), torch.zeros(3, H, 700)], 2)
    check_mass(got, mass64(q, lse, ks, 8, lens, full, n_new, decay=0.25), 0.0)
