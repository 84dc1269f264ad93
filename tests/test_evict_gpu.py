"""Eviction from the cache by accumulated attention weight against plain forms: the weights' sums
in 64 bits (bounds below), which tokens are kept and what is moved exactly.

Bound of a sum.  A score of D products accumulated in fp32 is off by at most (D + 8) 2^-23 of the sum
of its terms' magnitudes |q| (|m| + s u) times the scale; in log2 units, and less the row's lse, two
products and a difference round, 2^-22 (|score| + |lse|) together; the exponential is off by 2^-22.  With e
the sum of these a row's weight p is off by p (exp(e) - 1), and R of them, and what was there before, add
(R + 8) 2^-23 of the total."""
import math

import pytest
import torch

import paper_2603_29494_amd as va
import window_reference as ref
from test_cache_gpu import fresh_cache, int32, paged, rows

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23


def mass64(q, lse, k, bits, lens, mass, n_new=None, window=1 << 30, sinks=0, scale=0.0, decay=1.0,
           hidden=None):
    """[B, H] lists of sums of the tokens below lens, and their bounds; k[b] [H, lens[b], D] bf16."""
    q, lse = q.cpu().double(), lse.cpu().double()
    B, Hq, n, D = q.shape
    scale = scale or D ** -0.5
    out = []
    for b in range(B):
        L = int(lens[b])
        nb = n if n_new is None else min(max(int(n_new[b]), 0), n)
        H = k[b].shape[0]
        p = torch.arange(nb) + L - nb
        see = ref.sees(p, torch.arange(L), window, sinks, True, L)
        if hidden is not None:
            see = see & ~hidden[b][None, :]
        for h in range(H):
            u, m, s = ref.quantise(k[b][h].cpu(), bits)
            m, su = ref.spread(m), ref.spread(s) * u.reshape(L, D)
            w, e, R = torch.zeros(L, dtype=torch.float64), torch.zeros(L, dtype=torch.float64), 0
            for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                x, l = q[b, hq, :nb], lse[b, hq, :nb, None]
                y = (x @ (m + su).t()) * scale
                err = (x.abs() @ (m.abs() + su).t()) * scale * (D + 8) * STEP
                there = see & (l > -math.inf)
                l = torch.where(l > -math.inf, l, torch.zeros_like(l))
                pr = torch.exp(y - l).masked_fill(~there, 0.0)
                er = err + 2 * STEP * (y.abs() + l.abs()) + 2 * STEP
                w += pr.sum(0)
                e += (pr * torch.expm1(er).masked_fill(~there, 0.0)).sum(0)
                R += nb
            old = torch.zeros(L, dtype=torch.float64)
            if mass is not None:
                old[:max(0, L - nb)] = decay * mass[b, h, :max(0, L - nb)].cpu().double()
            total = w + old
            out.append((b, h, L, total, e + (R + 8) * STEP * total.abs() + 1e-37))
    return out


def check_mass(got, refs, untouched=None):
    for b, h, L, total, bound in refs:
        x = got[b, h, :L].cpu().double()
        over = ((x - total).abs() - bound)
        assert not over.isnan().any(), (b, h)
        assert over.max() <= 0, (b, h, over.max(), over.argmax())
        if untouched is not None:
            assert (got[b, h, L:] == untouched).all()


def setup(D, bits, page, lens, Hkv, group, n, seed=0, n_new=None, window=None, sinks=0, drop=None):
    """A filled cache, the last rows' q, and lse from attention over it."""
    ks = [rows(seed + 10 * b, Hkv, L, D) + rows(99, Hkv, 1, D, scale=2.0)
          for b, L in enumerate(lens)]
    table, pages = paged(lens, page, seed)
    cache = fresh_cache(pages, Hkv, D, page, bits)
    for b, L in enumerate(lens):
        if L:
            va.cache_write(cache, ks[b][None], ks[b][None], table[b:b + 1], int32([L]))
    if drop is not None:
        table[drop[0], drop[1]] = -1
    q = rows(seed + 5, len(lens), Hkv * group, n, D)
    _, lse = va.cache_attn(q, cache, table, int32(lens), n_new=n_new, window=window, sinks=sinks,
                           return_lse=True)
    return ks, cache, table, q, lse


@pytest.mark.parametrize("D,bits,page", [(128, 4, 64), (64, 4, 32), (128, 8, 32), (64, 8, 128)])
@pytest.mark.parametrize("group,n", [(1, 1), (7, 1), (4, 4), (5, 5), (1, 33), (7, 40), (2, 300),
                                     (8, 260), (5, 9), (16, 4), (1, 79), (9, 9)])
def test_mass(gpu, D, bits, page, group, n):
    lens = [max(n, L) for L in (1, 33, 700)]
    ks, cache, table, q, lse = setup(D, bits, page, lens, 2, group, n)
    M = table.shape[1] * page
    old = torch.rand(3, 2, M, generator=torch.Generator().manual_seed(1)).cuda()
    out = torch.full((3, 2, M), -7.0, device="cuda")
    got = va.cache_mass(q, lse, cache, table, int32(lens), mass=old, out=out)
    torch.cuda.synchronize()
    check_mass(got, mass64(q, lse, ks, bits, lens, old), -7.0)
    # without what was there; and in place, with a decay
    check_mass(va.cache_mass(q, lse, cache, table, int32(lens)),
               mass64(q, lse, ks, bits, lens, None), 0.0)
    again = old.clone()
    va.cache_mass(q, lse, cache, table, int32(lens), mass=again, decay=0.75, out=again)
    check_mass(again, mass64(q, lse, ks, bits, lens, old, decay=0.75))
    for b, L in enumerate(lens):
        assert torch.equal(again[b, :, L:], old[b, :, L:])


@pytest.mark.parametrize("group,n", [(7, 1), (4, 3), (3, 70), (8, 200), (3, 9), (13, 5),
                                     (5, 16)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (33, 5), (100, 64)])
def test_mass_window_padding_and_missing_pages(gpu, group, n, window, sinks):
    lens, n_new = [n + 400, n + 3, 2, 300], int32([n, 1, n + 9, 0])
    lens = [max(1, L) for L in lens]
    real = [min(max(int(x), 0), n) for x in n_new.tolist()]
    ks, cache, table, q, lse = setup(64, 4, 32, lens, 3, group, n, 3, n_new, window, sinks,
                                     drop=(0, 1))
    lse = lse.clone()
    for b in range(4):
        lse[b, :, real[b]:] = math.nan   # rows that are not there
    hidden = [torch.zeros(L, dtype=torch.bool) for L in lens]
    hidden[0][32:64] = True
    M = 333                              # neither a multiple of anything nor all tokens
    old = torch.rand(4, 3, M, generator=torch.Generator().manual_seed(2)).cuda()
    for inplace in (False, True):
        out = old.clone() if inplace else torch.full_like(old, -7.0)
        got = va.cache_mass(q, lse, cache, table, int32(lens), mass=out if inplace else old,
                            n_new=n_new, window=window, sinks=sinks, out=out)
        full = torch.cat([old.cpu(), torch.zeros(4, 3, 1000)], 2)
        refs = mass64(q, lse, ks, 4, lens, full, n_new, window, sinks, hidden=hidden)
        refs = [(b, h, min(L, M), t[:M], e[:M]) for b, h, L, t, e in refs]
        check_mass(got, refs)
        for b, L in enumerate(lens):
            assert torch.equal(got[b, :, L:], (old if inplace else torch.full_like(old, -7.0))[b, :, L:])


@pytest.mark.parametrize("group,n", [(3, 2), (3, 40), (8, 160)])
def test_mass_of_tokens_past_the_table(gpu, group, n):
    """Tokens that the table has no column for are held nowhere: what they had collected decays."""
    lens, held = [500, 700], 256
    ks, cache, table, _, _ = setup(64, 8, 32, lens, 2, group, n, 7)
    table = table[:, :held // 32].contiguous()
    q = rows(11, 2, 2 * group, n, 64)
    _, lse = va.cache_attn(q, cache, table, int32(lens), return_lse=True)
    hidden = [torch.arange(L) >= held for L in lens]
    old = torch.rand(2, 2, 640, generator=torch.Generator().manual_seed(3)).cuda()
    out = torch.full_like(old, -7.0)
    va.cache_mass(q, lse, cache, table, int32(lens), mass=old, decay=0.5, out=out)
    full = torch.cat([old.cpu(), torch.zeros(2, 2, 60)], 2)
    refs = mass64(q, lse, ks, 8, lens, full, decay=0.5, hidden=hidden)
    check_mass(out, [(b, h, min(L, 640), t[:640], e[:640]) for b, h, L, t, e in refs])
    assert (out[0, :, 500:] == -7.0).all()


def test_mass_adds_up_to_the_rows(gpu):
    """A row's weights sum to one: over all tokens the sums are the number of rows."""
    lens, n, group = [5000, 800], 20, 4
    ks, cache, table, q, lse = setup(128, 4, 64, lens, 2, group, n)
    got = va.cache_mass(q, lse, cache, table, int32(lens)).double().sum(2)
    assert (got - n * group).abs().max() <= n * group * 1e-4


def test_mass_rows_without_weight_and_nan_keys(gpu):
    """Rows whose lse is -inf add nothing; a NaN key reaches its own token's sum alone, and a hidden
    one not even that."""
    for n in (2, 40):
        ks, cache, table, q, lse = setup(128, 8, 32, [100], 1, 3, n)
        lse = lse.clone()
        lse[0, 1] = -math.inf
        check_mass(va.cache_mass(q, lse, cache, table, int32([100])),
                   mass64(q, lse, ks, 8, [100], None))
        bad = ks[0].clone()
        bad[0, 10, 3] = math.nan          # behind every row's window
        bad[0, 90 - n, 70] = math.inf     # seen
        va.cache_write(cache, bad[None], bad[None], table, int32([100]))
        got = va.cache_mass(q, lse, cache, table, int32([100]), window=50)
        clean = mass64(q, lse, ks, 8, [100], None, window=50)[0]
        x = got[0, 0, :100].cpu().double()
        assert x[90 - n].isnan() and x[10] == 0
        keep = torch.arange(100) != 90 - n
        assert ((x - clean[3]).abs() <= clean[4])[keep].all()


def keep_ref(mass, held, length, budget, sinks, recent):
    """Kept tokens of one head, from the definition."""
    order = []
    for j in held:
        x = float(mass[j])
        if j < sinks or j >= length - recent:
            order.append((0, 0.0, j))
        elif math.isnan(x):
            order.append((2, 0.0, j))
        else:
            order.append((1, -x, j))
    return sorted(j for _, _, j in sorted(order)[:budget])


@pytest.mark.parametrize("M,lens,budget,sinks,recent", [
    (64, [0, 1, 64], 1, 0, 0), (64, [5, 63, 64], 64, 3, 7), (100, [99, 100, 150], 40, 10, 30),
    (2000, [17, 1999, 900], 500, 0, 0), (9000, [8999, 1025, 70], 1000, 64, 128),
    (30000, [30000, 24577, 1], 7001, 4, 0), (16000, [16000, 8193, 15999], 4000, 0, 9),
    (70000, [70000, 40961, 1], 9001, 4, 70)])
@pytest.mark.parametrize("kind", ["spread", "ties", "special"])
def test_keep(gpu, M, lens, budget, sinks, recent, kind):
    H, page = 2, 32
    g = torch.Generator().manual_seed(M + budget)
    mass = torch.exp(3 * torch.randn(3, H, M, generator=g))
    if kind == "ties":
        mass = torch.randint(0, 3, (3, H, M), generator=g).float()
    if kind == "special":
        pick = torch.randint(0, 8, (3, H, M), generator=g)
        for i, x in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0, -1.5, 1e-40)):
            mass[pick == i] = x
    cols = -(-max(lens) // page)
    table = torch.arange(3 * cols).view(3, cols).int()
    table[0, cols // 2] = -1               # a page that is not held
    table[1, cols - 1] = 3 * cols + 5      # past the pages
    cache = va.cache_alloc(3 * cols, H, 64, page, 4)
    idx, kept = va.cache_keep(mass.cuda(), cache, table.cuda(), int32(lens), budget, sinks, recent)
    torch.cuda.synchronize()
    for b in range(3):
        held = [j for j in range(min(lens[b], M))
                if 0 <= int(table[b, j // page]) < 3 * cols]
        assert int(kept[b]) == min(budget, len(held))
        for h in range(H):
            want = keep_ref(mass[b, h].tolist(), held, lens[b], budget, sinks, recent)
            want += [-1] * (budget - len(want))
            assert idx[b, h].tolist() == want, (b, h)


@pytest.mark.parametrize("D,bits,page,to_page", [(128, 4, 64, 32), (64, 4, 32, 32), (128, 8, 32, 128),
                                                 (64, 8, 128, 64)])
def test_gather(gpu, D, bits, page, to_page):
    H, lens, budget = 3, [300, 40, 5, 900], 130
    k, v = rows(1, 4, H, 900, D), rows(2, 4, H, 900, D)
    table, pages = paged(lens, page)
    cache = fresh_cache(pages, H, D, page, bits)
    va.cache_write(cache, k, v, table, int32(lens), n_new=int32(lens))
    g = torch.Generator().manual_seed(4)
    kept = [min(budget, L) for L in lens]
    idx = torch.full((4, H, budget), -1, dtype=torch.int32)
    for b in range(4):
        for h in range(H):
            idx[b, h, :kept[b]] = torch.sort(torch.randperm(lens[b], generator=g)[:kept[b]])[0].int()
    idx[3, 1, :kept[3]] = torch.flip(idx[3, 1, :kept[3]], [0])   # any order
    idx[3, 2, 10:20] = 7                                         # the same token again
    mass = torch.rand(4, H, 900, generator=g)
    to_table, to_pages = paged(kept, to_page, 7)
    same_cache = to_page == page
    if same_cache:   # pages behind those that are read
        big = fresh_cache(pages + to_pages, H, D, page, bits)
        big.data[:cache.data.numel()] = cache.data
        cache, to, to_table = big, None, torch.where(to_table >= 0, to_table + pages, to_table)
    else:
        to = fresh_cache(to_pages, H, D, to_page, bits)
    before = cache.data.clone()
    moved = va.cache_gather(cache, table, idx.cuda(), int32(kept), to_table, to=to, mass=mass.cuda())
    dst = cache if to is None else to
    gk, gv = va.cache_read(dst, to_table, int32(kept), budget)
    sk, sv = va.cache_read(cache, table, int32(lens), 900)
    torch.cuda.synchronize()
    for b in range(4):
        n = kept[b]
        for h in range(H):
            at = idx[b, h, :n].long()
            assert torch.equal(gk[b, h, :n].cpu(), sk[b, h].cpu()[at])
            assert torch.equal(gv[b, h, :n].cpu(), sv[b, h].cpu()[at])
            assert torch.equal(moved[b, h, :n].cpu(), mass[b, h][at])
            assert (moved[b, h, n:] == 0).all()
    half = before.numel() if to is not None else pages * H * page * 2 * (D * bits // 8 + D // 16)
    assert torch.equal(cache.data[:half], before[:half])   # what is read stays


def test_gather_of_tokens_that_are_not_there(gpu):
    H, D, page = 1, 128, 32
    k = rows(1, 1, H, 100, D)
    table, pages = paged([100], page)
    cache = fresh_cache(pages + 2, H, D, page, 4)
    va.cache_write(cache, k, k, table, int32([100]))
    sk, _ = va.cache_read(cache, table, int32([100]), 100)
    table = table.clone()
    table[0, 1] = pages + 77
    idx = int32([[[3, -1, 40, 99, 128, 1 << 30, -2 ** 31, 0]]])
    to = torch.full((1, 1), pages, dtype=torch.int32, device="cuda")
    mass = torch.arange(100.0, device="cuda").view(1, 1, 100)
    moved = va.cache_gather(cache, table, idx, int32([99]), to, mass=mass)   # kept is clamped
    gk, gv = va.cache_read(cache, to, int32([8]), 8)
    there = torch.tensor([True, False, False, True, False, False, False, True])
    assert gk[0, 0, ~there].isnan().all() and gv[0, 0, ~there].isnan().all()
    assert torch.equal(gk[0, 0, there], sk[0, 0, [3, 99, 0]])
    want = torch.tensor([3.0, math.nan, 40.0, 99.0, math.nan, math.nan, math.nan, 0.0])
    assert torch.equal(moved[0, 0].cpu().nan_to_num(-1), want.nan_to_num(-1))
    # no page to take them, none kept: nothing is written
    before = cache.data.clone()
    for t, n in ((-1, 8), (pages + 2, 8), (pages, 0), (pages, -3)):
        va.cache_gather(cache, table, idx, int32([n]), torch.full_like(to, t))
    assert torch.equal(cache.data, before)


def test_a_layer_with_eviction(gpu):
    """Turned, written, attended, weighed, cut, and attended again, the last step as a graph that
    is replayed: what is kept attends as a cache of those tokens alone."""
    B, Hq, Hkv, D, page, budget = 2, 8, 2, 128, 32, 96
    lens = [200, 61]
    plan = va.rope_plan(D, layout="half")
    q, k = rows(1, B, Hq, 200, D), rows(2, B, Hkv, 200, D)
    v = rows(3, B, Hkv, 200, D)
    n_new = int32(lens)
    q, k = va.rope(plan, q, k, lens=n_new, n_new=n_new)
    table, pages = paged(lens, page)
    cache = fresh_cache(pages + 8, Hkv, D, page, 8)
    va.cache_write(cache, k, v, table, n_new, n_new=n_new)
    _, lse = va.cache_attn(q, cache, table, n_new, n_new=n_new, return_lse=True)
    mass = va.cache_mass(q, lse, cache, table, n_new, n_new=n_new)
    idx, kept = va.cache_keep(mass, cache, table, n_new, budget, sinks=4, recent=16)
    to = torch.full((B, 4), -1, dtype=torch.int32, device="cuda")
    to[0], to[1, :3] = torch.arange(pages, pages + 4), torch.arange(pages + 4, pages + 7)
    left = va.cache_gather(cache, table, idx, kept, to, mass=mass)
    assert kept.tolist() == [96, 61]
    for b in range(B):
        n = int(kept[b])
        assert torch.equal(left[b, :, :n], mass[b].gather(1, idx[b, :, :n].long()))
        assert idx[b, :, :4].tolist() == [[0, 1, 2, 3]] * Hkv
    # a new token at its own position, behind the kept ones; M grows with the pages
    state = torch.zeros(B, Hkv, 128, device="cuda")
    state[:, :, :budget] = left
    q1, k1, v1 = rows(4, B, Hq, 1, D), rows(5, B, Hkv, 1, D), rows(6, B, Hkv, 1, D)
    pos, held = int32([[200], [61]]), kept + 1
    o1 = torch.zeros_like(q1)
    sk, sv = va.cache_read(cache, to, kept, 127)
    plain_q, plain_k = va.rope(plan, q1, k1, pos=pos)

    def step():
        a, c = va.rope(plan, q1, k1, pos=pos)
        va.cache_write(cache, c, v1, to, held)
        _, l1 = va.cache_attn(a, cache, to, held, out=o1, return_lse=True)
        va.cache_mass(a, l1, cache, to, held, mass=state, out=state)
        return l1
    first = state.clone()
    step()
    got, weights = o1.clone(), state.clone()
    kk = [torch.cat([sk[b, :, :int(kept[b])], plain_k[b]], 1) for b in range(B)]
    vv = [torch.cat([sv[b, :, :int(kept[b])], v1[b]], 1) for b in range(B)]
    for b in range(B):
        # sk, sv are bf16 roundings of what is held, and the new token's rows of its own codes:
        # compare with attention over what is read back, whose scores are off by |q| |k| 2^-8 / 8
        n = int(held[b])
        rk, rv = va.cache_read(cache, to, held, 128)
        x = plain_q[b].double().cpu().view(Hkv, 4, D) @ rk[b, :, :n].double().cpu().transpose(1, 2)
        w = torch.softmax(x / D ** 0.5, -1)
        want = (w @ rv[b, :, :n].double().cpu()).view(Hq, D)
        e = (plain_q[b].double().cpu().abs().view(Hkv, 4, D)
             @ rk[b, :, :n].double().cpu().abs().transpose(1, 2)).amax(-1) / D ** 0.5 * 2 ** -8
        slack = (2 * e.view(Hq, 1) + 3 * 2 ** -8) * (w @ rv[b, :, :n].double().cpu().abs()).view(Hq, D)
        assert ((got[b, :, 0].double().cpu() - want).abs() <= slack + 2 ** -8 * want.abs()).all()
        # one token's weights of four heads add up to four
        gain = (weights[b].double() - first[b].double()).sum(1)
        assert (gain - 4).abs().max() < 1e-3
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        state.copy_(first)
        o1.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o1, got) and torch.equal(state, weights)


@pytest.mark.parametrize("D,bits,page", [(128, 4, 64), (64, 8, 32)])
@pytest.mark.parametrize("start", [0, 5, 70])
def test_reading_back_whole(gpu, D, bits, page, start):
    """Outputs that the call makes are 0 wherever no token is held, whatever memory they get."""
    lens = [100, 1, 0, 193]
    k = rows(1, 4, 2, 193, D)
    table, pages = paged(lens, page)
    cache = fresh_cache(pages, 2, D, page, bits)
    va.cache_write(cache, k, k, table, int32(lens), n_new=int32(lens))
    table[3, 1] = -1
    for n in (1, 33, 250):
        want = [torch.zeros(4, 2, n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        va.cache_read(cache, table, int32(lens), n, start=start, out=tuple(want))
        junk = [torch.full_like(want[0], 7.0) for _ in range(2)]
        del junk
        for a, b in zip(va.cache_read(cache, table, int32(lens), n, start=start), want):
            assert torch.equal(a, b)


def test_calls_at_once_give_what_they_give_alone(gpu):
    ks, cache, table, q, lse = setup(128, 4, 64, [9000, 3000], 4, 7, 1)
    lens = int32([9000, 3000])
    mass = va.cache_mass(q, lse, cache, table, lens)
    idx, kept = va.cache_keep(mass, cache, table, lens, 2000, 16, 100)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            m = va.cache_mass(q, lse, cache, table, lens)
            outs.append((m, *va.cache_keep(m, cache, table, lens, 2000, 16, 100)))
    torch.cuda.synchronize()
    for m, i, n in outs:
        assert torch.equal(m, mass) and torch.equal(i, idx) and torch.equal(n, kept)


def test_replayed_chunks_and_long_rows(gpu):
    """Graphs that share a workspace, of calls of several launches, follow the lengths on the
    device; between the replays the same calls run eagerly."""
    ks, cache, table, q, _ = setup(64, 4, 32, [700, 300], 2, 4, 160)
    other = rows(77, *q.shape)
    lens, n_new = int32([700, 300]), int32([160, 160])
    lse = torch.full(q.shape[:3], 6.0, device="cuda")
    M = 40960
    long = fresh_cache(2 * M // 64, 1, 64, 64, 4)
    pages = torch.randperm(2 * M // 64, generator=torch.Generator().manual_seed(5))
    pages = pages.to(torch.int32).view(2, -1).cuda()
    mass = torch.rand(2, 1, M, generator=torch.Generator().manual_seed(6)).cuda()
    held = int32([M, 33000])
    need = max(va.cache_mass_workspace_bytes(q, cache),
               va.cache_keep_workspace_bytes(mass, long, pages.shape[1]))
    assert va.cache_keep_workspace_bytes(mass, long, pages.shape[1]) > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros(2, 2, table.shape[1] * 32, device="cuda") for _ in range(2)]

    def weights(x, out):
        return va.cache_mass(x, lse, cache, table, lens, n_new=n_new, out=out, workspace=ws)
    graphs, kept = [], []
    for x, out in zip((q, other), outs):
        weights(x, out)
        va.cache_keep(mass, long, pages, held, 500, 4, 64, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            weights(x, out)
            kept.append(va.cache_keep(mass, long, pages, held, 500, 4, 64, workspace=ws))
    for a, b, long_lens in (((700, 300), (160, 160), (M, 33000)), ((161, 0), (160, 0), (0, 1)),
                            ((500, 299), (3, 160), (40000, 501)), ((700, 300), (160, 160), (M, M))):
        lens.copy_(int32(a)), n_new.copy_(int32(b)), held.copy_(int32(long_lens))
        for i, x in enumerate((q, other)):
            outs[i].fill_(-3.0)
            want = weights(x, torch.full_like(outs[i], -3.0))
            idx, n = va.cache_keep(mass, long, pages, held, 500, 4, 64, workspace=ws)
            torch.cuda.synchronize()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want)
            assert torch.equal(kept[i][0], idx) and torch.equal(kept[i][1], n)
            assert n.tolist() == [min(500, L) for L in long_lens]
            for s in range(2):
                ref_idx = keep_ref(mass[s, 0].tolist(), range(long_lens[s]), long_lens[s], 500, 4, 64)
                assert idx[s, 0, :len(ref_idx)].tolist() == ref_idx
