"""The quantised, paged key/value cache and attention over it against plain 64-bit forms; bounds
in window_reference.  What is written and read back is equal bit for bit (the format is defined
by its fp32 steps)."""
import math

import pytest
import torch

import paper_2603_29494_amd as va
import window_reference as ref

pytestmark = pytest.mark.gpu


def rows(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).bfloat16().cuda()


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def paged(lens, page, seed=0, spare=2, cols=None):
    """A table of shuffled pages for sequences of these lengths, and how many there are."""
    per = [-(-L // page) for L in lens]
    pages = sum(per) + spare
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    table = torch.full((len(lens), cols or max(1, max(per))), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(per):
        table[b, :c] = ids[at:at + c]
        at += c
    return table.cuda(), pages


def fresh_cache(pages, H, D, page, bits):
    """Memory that reads NaN everywhere it has not been written."""
    c = va.cache_alloc(pages, H, D, page, bits)
    c.data.fill_(0xFF)
    return c


def bf16_value(x, bits):
    u, m, s = ref.quantise(x.cpu(), bits)
    return (ref.spread(m).float() + (ref.spread(s) * u).float()).bfloat16()


def same(a, b):
    """Equal bits, any NaN equal to any."""
    a, b = a.cpu(), b.cpu()
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0, 1e38, -1e38),
                                                             b.nan_to_num(0.0, 1e38, -1e38))


FORMATS = [(128, 4, 64), (64, 4, 32), (128, 8, 32), (64, 8, 1024)]


@pytest.mark.parametrize("D,bits,page", FORMATS)
@pytest.mark.parametrize("lens", [[1], [31, 32, 33], [100, 1, 257, 64]])
def test_round_trip_is_the_format(gpu, lens, D, bits, page):
    H, n = 3, max(lens)
    k, v = rows(1, len(lens), H, n, D, scale=2.0), rows(2, len(lens), H, n, D)
    k += rows(3, 1, H, 1, D, scale=4.0)
    table, pages = paged(lens, page)
    cache = fresh_cache(pages, H, D, page, bits)
    va.cache_write(cache, k, v, table, int32(lens), n_new=int32(lens))
    gk, gv = va.cache_read(cache, table, int32(lens), n)
    torch.cuda.synchronize()
    for b, L in enumerate(lens):
        assert same(gk[b, :, :L], bf16_value(k[b, :, :L], bits))
        assert same(gv[b, :, :L], bf16_value(v[b, :, :L], bits))
        assert (gk[b, :, L:] == 0).all() and (gv[b, :, L:] == 0).all()


@pytest.mark.parametrize("D,bits,page", FORMATS)
def test_special_groups(gpu, D, bits, page):
    """Constant, zero, tiny, subnormal, huge and non-finite groups."""
    x = rows(4, 1, 1, 40, D)
    x[0, 0, 0] = 0.0
    x[0, 0, 1] = 3.5
    x[0, 0, 2] *= 1e-30
    x[0, 0, 3] *= 1e-37
    x[0, 0, 4] = torch.finfo(torch.bfloat16).smallest_normal / 8
    x[0, 0, 5] *= 1e36
    x[0, 0, 6, 7] = math.inf
    x[0, 0, 7, D - 1] = -math.inf
    x[0, 0, 8, 0] = math.nan
    x[0, 0, 9, 0], x[0, 0, 9, 1] = 3.3e38, -3.3e38     # a range past fp32
    x[0, 0, 10, 0] = 1e5                                # one outlier
    x[0, 0, 11] = torch.arange(D).bfloat16().cuda() / 2   # ties
    x[0, 0, 12] = -x[0, 0, 11]
    table, pages = paged([40], page)
    cache = fresh_cache(pages, 1, D, page, bits)
    va.cache_write(cache, x, x.flip(-1), table, int32([40]))
    gk, gv = va.cache_read(cache, table, int32([40]), 40)
    assert same(gk, bf16_value(x, bits))
    assert same(gv, bf16_value(x.flip(-1), bits))
    assert gk[0, 0, 8, :64].isnan().all() and gk[0, 0, 9, :64].isnan().all()


@pytest.mark.parametrize("D,bits,page", FORMATS)
def test_token_by_token_is_the_same_cache(gpu, D, bits, page):
    """Tokens appended one by one, two and three at a time leave what one call leaves, byte for
    byte, and nothing else is touched."""
    H, lens = 2, [70, 35]
    k, v = rows(5, 2, H, 70, D), rows(6, 2, H, 70, D)
    table, pages = paged(lens, page)
    a, b = fresh_cache(pages, H, D, page, bits), fresh_cache(pages, H, D, page, bits)
    va.cache_write(a, k, v, table, int32(lens), n_new=int32(lens))
    at = [0, 0]
    step = 0
    while at != lens:
        take = [min((1, 2, 3)[step % 3], L - x) for x, L in zip(at, lens)]
        kn, vn = (torch.zeros(2, H, 3, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        for s in range(2):
            kn[s, :, :take[s]] = k[s, :, at[s]:at[s] + take[s]]
            vn[s, :, :take[s]] = v[s, :, at[s]:at[s] + take[s]]
        at = [x + t for x, t in zip(at, take)]
        va.cache_write(b, kn, vn, table, int32(at), n_new=int32(take))
        step += 1
    assert torch.equal(a.data, b.data)


@pytest.mark.parametrize("D,bits,page", FORMATS[:2])
def test_holes_and_lengths_past_the_table(gpu, D, bits, page):
    """Entries that name no page are not written and not read; nor are tokens past the table, nor
    rows at a position below 0."""
    H, L = 2, 5 * page
    k, v = rows(7, 1, H, L, D), rows(8, 1, H, L, D)
    table, pages = paged([3 * page], page, cols=4)
    table[0, 1] = -1
    table[0, 3] = pages          # past the last page
    cache = fresh_cache(pages, H, D, page, bits)
    before = cache.data.clone()
    va.cache_write(cache, k, v, table, int32([L]))
    out = tuple(torch.full((1, H, L, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    va.cache_read(cache, table, int32([L]), L, out=out)
    for x, got in ((k, out[0]), (v, out[1])):
        for c in range(5):
            sl = slice(c * page, (c + 1) * page)
            if c in (0, 2):
                assert same(got[:, :, sl], bf16_value(x[:, :, sl], bits))
            else:
                assert (got[:, :, sl] == 5.0).all()
    per = cache.data.numel() // pages
    used = {int(table[0, 0]), int(table[0, 2])}
    for i in range(pages):
        if i not in used:
            assert torch.equal(cache.data[i * per:(i + 1) * per], before[i * per:(i + 1) * per])
    # more new rows than tokens: the last ones are kept
    cache.data.copy_(before)
    va.cache_write(cache, k[:, :, :40], v[:, :, :40], table, int32([9]))
    gk, _ = va.cache_read(cache, table, int32([9]), 9)
    assert same(gk, bf16_value(k[:, :, 31:40], bits))


@pytest.mark.parametrize("start,n", [(0, 1), (31, 2), (40, 33), (64, 100), (150, 500)])
def test_read_of_a_part(gpu, start, n):
    k, v = rows(9, 2, 2, 200, 128), rows(10, 2, 2, 200, 128)
    table, pages = paged([200, 90], 32)
    cache = fresh_cache(pages, 2, 128, 32, 4)
    va.cache_write(cache, k, v, table, int32([200, 90]), n_new=int32([200, 90]))
    gk, gv = va.cache_read(cache, table, int32([200, 90]), n, start=start)
    for b, L in enumerate((200, 90)):
        m = max(0, min(n, L - start))
        assert same(gk[b, :, :m], bf16_value(k[b, :, start:start + m], 4))
        assert same(gv[b, :, :m], bf16_value(v[b, :, start:start + m], 4))
        assert (gk[b, :, m:] == 0).all()


def filled(seed, lens, H, D, page, bits, table=None, pages=None):
    """A cache of random sequences and the rows it was written from."""
    if table is None:
        table, pages = paged(lens, page, seed)
    cache = fresh_cache(pages, H, D, page, bits)
    ks, vs = [], []
    for b, L in enumerate(lens):
        k = rows(seed + 10 * b, 1, H, max(L, 1), D) + rows(seed, 1, H, 1, D, scale=2.0)
        v = rows(seed + 10 * b + 1, 1, H, max(L, 1), D) + 0.5
        if L:
            va.cache_write(cache, k, v, table[b:b + 1], int32([L]))
        ks.append(k[0, :, :L].cpu())
        vs.append(v[0, :, :L].cpu())
    return cache, table, ks, vs


def attn_case(seed, lens, Hq, H, n, D, bits, page, window=None, sinks=0, n_new=None, scale=0.0):
    cache, table, ks, vs = filled(seed, lens, H, D, page, bits)
    q = rows(seed + 7, len(lens), Hq, n, D, scale=1.5)
    out = torch.full_like(q, 9.0)
    o, lse = va.cache_attn(q, cache, table, int32(lens), None if n_new is None else int32(n_new),
                           window, sinks, scale, out, True)
    torch.cuda.synchronize()
    r = ref.cache_attn(q, ks, vs, bits, lens, n_new, window or 1 << 30, sinks, scale)
    ref.check(o, lse, r, f"{lens} {Hq}/{H} n={n} D={D} {bits} bits window={window} sinks={sinks}")
    assert (o.cpu()[torch.isnan(r[1])] == 9.0).all()      # padded rows stay


@pytest.mark.parametrize("D,bits,page", FORMATS)
@pytest.mark.parametrize("lens", [[1], [31, 32, 33, 64, 65], [700, 5]])
@pytest.mark.parametrize("Hq,H", [(1, 1), (7, 1), (16, 2), (20, 1), (34, 1)])
def test_one_token(gpu, Hq, H, lens, D, bits, page):
    attn_case(100, lens, Hq, H, 1, D, bits, page)


@pytest.mark.parametrize("D,bits,page", FORMATS)
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 3), (1, 0), (33, 64)])
@pytest.mark.parametrize("n,Hq,H", [(2, 4, 2), (5, 7, 1), (40, 3, 1), (70, 2, 2)])
def test_several_tokens(gpu, n, Hq, H, window, sinks, D, bits, page):
    attn_case(200, [300, 70], Hq, H, n, D, bits, page, window, sinks)


@pytest.mark.parametrize("D,bits,page", FORMATS)
@pytest.mark.parametrize("window,sinks", [(None, 0), (1500, 70), (64, 1)])
def test_long_sequences_split(gpu, window, sinks, D, bits, page):
    attn_case(300, [9001, 2048, 33], 8, 2, 1, D, bits, page, window, sinks, scale=0.05)


@pytest.mark.parametrize("lens,n_new", [([50, 3, 0, 20], [4, 3, 0, 9]), ([5, 2, 1, 0], [1, 5, 0, 3])])
def test_padded_and_short_batches(gpu, lens, n_new):
    """Rows past n_new stay as they were; rows at positions below 0 see nothing."""
    attn_case(400, lens, 6, 3, 5, 128, 4, 32, None, 0, n_new)
    attn_case(401, lens, 6, 3, 5, 64, 8, 32, 2, 1, n_new)


@pytest.mark.parametrize("n,window,sinks", [(1, None, 0), (3, 50, 40)])
def test_pages_that_are_not_there(gpu, n, window, sinks):
    """Tokens of holes and past the table are not seen; a row that sees nothing is 0, -inf."""
    page, D, bits, lens = 32, 128, 4, [150, 90, 200]
    table, pages = paged([150, 90, 160], page, 3, cols=5)   # the last has 40 tokens too many
    cache, table, ks, vs = filled(500, lens, 2, D, page, bits, table, pages)
    table[0, 1], table[0, 4] = -1, pages + 5
    table[1, :] = -7
    hidden = [torch.zeros(L, dtype=torch.bool) for L in lens]
    hidden[0][32:64] = hidden[0][128:] = True
    hidden[1][:] = True
    hidden[2][160:] = True
    q = rows(507, 3, 4, n, D, scale=1.5)
    o, lse = va.cache_attn(q, cache, table, int32(lens), window=window, sinks=sinks, return_lse=True)
    ref.check(o, lse, ref.cache_attn(q, ks, vs, bits, lens, None, window or 1 << 30, sinks, 0.0,
                                     hidden))
    assert (lse[1] == -math.inf).all()


@pytest.mark.parametrize("n", [4, 40])
@pytest.mark.parametrize("D,bits", [(128, 4), (64, 8)])
def test_hidden_tokens_never_reach_a_row(gpu, D, bits, n):
    """NaN groups outside a row's window change nothing; inside they make it NaN."""
    L, window = 300, 60
    table, pages = paged([L], 32)
    k, v = rows(601, 1, 1, L, D), rows(602, 1, 1, L, D)
    q = rows(603, 1, 2, n, D)
    lens = int32([L])

    def run(kk, vv):
        cache = fresh_cache(pages, 1, D, 32, bits)
        va.cache_write(cache, kk, vv, table, lens)
        return va.cache_attn(q, cache, table, lens, window=window, sinks=1)
    clean = run(k, v)
    at = L - n - window + 3     # row r sees from L - n + r - window + 1 on: the first three do
    seen = torch.tensor([L - n + r - window < at for r in range(n)]).cuda()
    assert seen.any() and not seen.all()
    for bad in ("k", "v"):
        kk, vv = k.clone(), v.clone()
        (kk if bad == "k" else vv)[0, 0, at, 1] = math.nan
        (kk if bad == "k" else vv)[0, 0, 50] = math.inf
        o = run(kk, vv)
        assert torch.equal(o[:, :, ~seen], clean[:, :, ~seen]), bad
        assert o[:, :, seen][..., :64].isnan().all(), bad


def test_large_scores(gpu):
    """References move by hundreds along a sequence; no weight overflows."""
    L, D = 3000, 128
    table, pages = paged([L], 64)
    k, v = rows(701, 1, 1, L, D), rows(702, 1, 1, L, D)
    for ramp in (torch.linspace(0.1, 30, L), torch.linspace(30, 0.1, L)):
        kk = (k * ramp.bfloat16().cuda()[None, None, :, None])
        cache = fresh_cache(pages, 1, D, 64, 4)
        va.cache_write(cache, kk, v, table, int32([L]))
        q = rows(703, 1, 4, 1, D)
        o, lse = va.cache_attn(q, cache, table, int32([L]), return_lse=True)
        ref.check(o, lse, ref.cache_attn(q, [kk[0].cpu()], [v[0].cpu()], 4, [L]))


def test_shared_pages(gpu):
    """Sequences that share a prompt's pages read them as if each had its own."""
    page, D = 64, 128
    k, v = rows(801, 1, 2, 128, D), rows(802, 1, 2, 128, D)
    cache = fresh_cache(4, 2, D, page, 4)
    va.cache_write(cache, k, v, torch.tensor([[2, 0]], dtype=torch.int32).cuda(), int32([128]))
    table = torch.tensor([[2, 0, 1], [2, 0, 3]], dtype=torch.int32).cuda()
    kn, vn = rows(803, 2, 2, 3, D), rows(804, 2, 2, 3, D)
    lens = int32([131, 130])
    va.cache_write(cache, kn, vn, table, lens, n_new=int32([3, 2]))
    q = rows(805, 2, 4, 1, D)
    o, lse = va.cache_attn(q, cache, table, lens, return_lse=True)
    ks = [torch.cat([k[0], kn[0]], 1).cpu(), torch.cat([k[0], kn[1, :, :2]], 1).cpu()]
    vs = [torch.cat([v[0], vn[0]], 1).cpu(), torch.cat([v[0], vn[1, :, :2]], 1).cpu()]
    ref.check(o, lse, ref.cache_attn(q, ks, vs, 4, [131, 130]))


def test_layouts(gpu):
    """Rows of a packed projection, written and attended to without a copy, into a wider output."""
    B, Hq, H, D = 3, 6, 2, 128
    proj = rows(901, B, (Hq + 2 * H) * D)
    q, k, v = (t.view(B, -1, 1, D) for t in proj.split([Hq * D, H * D, H * D], 1))
    lens = [40, 1, 97]
    cache, table, ks, vs = filled(902, lens, H, D, 32, 4)
    va.cache_write(cache, k, v, table, int32(lens))
    for b, L in enumerate(lens):
        ks[b][:, L - 1], vs[b][:, L - 1] = k[b, :, 0].cpu(), v[b, :, 0].cpu()
    buf = torch.zeros(B, 1, Hq + 1, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    o, lse = va.cache_attn(q, cache, table, int32(lens), out=buf[:, 1:], return_lse=True)
    ref.check(o, lse, ref.cache_attn(q, ks, vs, 4, lens))
    assert (buf[:, 0] == 0).all()


def test_step_on_a_stream_and_in_a_replayed_graph(gpu):
    """A decoding step (write, attend) captured once and replayed as lens, table and inputs
    change, each replay against the same step run eagerly on a copy."""
    B, Hq, H, D, page = 3, 8, 2, 128, 32
    lens0 = [400, 31, 2200]
    table, pages = paged([L + 40 for L in lens0], page)
    cache, table, _, _ = filled(950, lens0, H, D, page, 4, table, pages)
    twin = va.Cache(cache.data.clone(), cache.pages, H, D, page, 4)
    lens = int32(lens0)
    q, k, v = rows(1, B, Hq, 1, D), rows(2, B, H, 1, D), rows(3, B, H, 1, D)
    out = torch.zeros_like(q)
    ws = torch.empty(max(16, va.cache_attn_workspace_bytes(q, cache, table.shape[1])),
                     dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o = va.cache_attn(q, cache, table, lens)
    side.synchronize()
    assert torch.equal(o, va.cache_attn(q, cache, table, lens))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        va.cache_write(cache, k, v, table, lens)
        va.cache_attn(q, cache, table, lens, out=out, workspace=ws)
    for step in range(4):
        lens += 1
        for t, s in ((q, 10), (k, 20), (v, 30)):
            t.copy_(rows(s + step, *t.shape))
        graph.replay()
        va.cache_write(twin, k, v, table, lens)
        want = va.cache_attn(q, twin, table, lens)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
        assert torch.equal(cache.data, twin.data), step


@pytest.mark.parametrize("bits", [4, 8])
def test_a_model_layer_in_use(gpu, bits):
    """A prompt through the vector-sparse layer and a window layer, its K and V into the cache,
    then a drafted pair and single tokens: each step against 64 bits over what the cache holds;
    then the prompt read back for a selection over it."""
    Hq, H, D, N, page, window, sinks = 8, 2, 128, 500, 64, 128, 4
    q, k, v = rows(1, 1, Hq, N, D), rows(2, 1, H, N, D), rows(3, 1, H, N, D)
    table, pages = paged([N + 8], page)
    cache = fresh_cache(pages, H, D, page, bits)
    idx, cnt = va.select(q, k, 64, "topk", 0.2, True)
    va.sparse_attn(q, k, v, idx, cnt, 64, True)
    o, lse = va.window_attn(q, k, v, window, sinks, True, return_lse=True)
    ref.check(o, lse, ref.window_attn(q, k, v, window, sinks, True))
    lens = int32([N])
    va.cache_write(cache, k, v, table, lens)
    L = N
    for n in (2, 1, 1, 4):
        kn, vn, qn = rows(L, 1, H, n, D), rows(L + 1, 1, H, n, D), rows(L + 2, 1, Hq, n, D)
        k, v = torch.cat([k, kn], 2), torch.cat([v, vn], 2)
        L += n
        lens += n
        va.cache_write(cache, kn, vn, table, lens)
        for w, s in ((None, 0), (window, sinks)):
            o, lse = va.cache_attn(qn, cache, table, lens, window=w, sinks=s, return_lse=True)
            ref.check(o, lse, ref.cache_attn(qn, [k[0].cpu()], [v[0].cpu()], bits, [L], None,
                                             w or 1 << 30, s))
    gk, gv = va.cache_read(cache, table, lens, N)
    assert same(gk, bf16_value(k[:, :, :N], bits)) and same(gv, bf16_value(v[:, :, :N], bits))
    idx, cnt = va.select(q, gk, 64, "topk", 0.2, True)
    assert va.check_lists(idx, cnt, N) == 0


@pytest.mark.parametrize("D,bits,page", FORMATS)
@pytest.mark.parametrize("n,Hq,H,window,sinks", [(33, 1, 1, None, 0), (150, 2, 1, None, 0),
                                                 (64, 7, 1, 100, 40), (300, 1, 1, 1, 5)])
def test_chunks_of_a_prompt(gpu, n, Hq, H, window, sinks, D, bits, page):
    """More than 32 rows per key/value head, over sequences that end in a block's middle; split
    over the keys where they are long."""
    attn_case(800, [n + 1, 2500, n], Hq, H, n, D, bits, page, window, sinks)


@pytest.mark.parametrize("scale", [2.0 ** -60, 1e-6, 3e4, 2.0 ** 60])
@pytest.mark.parametrize("n", [1, 20, 50])
def test_magnitudes(gpu, n, scale):
    """Values far from 1, in K against 1 / scale in Q, in V, and growing along a sequence."""
    L, D = 700, 128
    table, pages = paged([L], 64)
    g = torch.linspace(-6, 0, L).exp2().bfloat16().cuda()[None, None, :, None]
    k, v = rows(851, 1, 1, L, D) * scale, rows(852, 1, 1, L, D) * scale * g
    q = rows(853, 1, 2, n, D) / scale
    cache = fresh_cache(pages, 1, D, 64, 4)
    va.cache_write(cache, k, v, table, int32([L]))
    o, lse = va.cache_attn(q, cache, table, int32([L]), return_lse=True)
    ref.check(o, lse, ref.cache_attn(q, [k[0].cpu()], [v[0].cpu()], 4, [L]))


@pytest.mark.parametrize("n", [1, 12, 50])
def test_zero_keys_and_tiny_queries(gpu, n):
    """Blocks of zeros under queries near 0: scores of 0 and masks that stay masks."""
    L, D = 200, 64
    table, pages = paged([L], 32)
    cache = fresh_cache(pages, 1, D, 32, 4)
    k, v = torch.zeros(1, 1, L, D, dtype=torch.bfloat16, device="cuda"), rows(861, 1, 1, L, D)
    va.cache_write(cache, k, v, table, int32([L]))
    q = rows(862, 1, 2, n, D, scale=1e-6)
    q[:, 1] = 0
    o, lse = va.cache_attn(q, cache, table, int32([L]), window=70, sinks=2, scale=1e-6,
                           return_lse=True)
    ref.check(o, lse, ref.cache_attn(q, [k[0].cpu()], [v[0].cpu()], 4, [L], None, 70, 2, 1e-6))


def test_many_sequences(gpu):
    """More row tiles than the lengths are dealt out for: one chunk per sequence."""
    lens = [(37 * i) % 211 for i in range(300)]
    attn_case(870, lens, 2, 1, 1, 64, 4, 32)


def test_two_calls_at_once(gpu):
    """Calls on two streams, each with a workspace of its own."""
    lens = [5000, 300]
    cache, table, ks, vs = filled(880, lens, 2, 128, 64, 4)
    qs = [rows(881 + i, 2, 8, 1, 128) for i in range(2)]
    want = [va.cache_attn(q, cache, table, int32(lens)) for q in qs]
    t = int32(lens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(va.cache_attn(qs[i], cache, table, t))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


@pytest.mark.parametrize("D,bits", [(128, 4), (64, 4), (128, 8), (64, 8)])
@pytest.mark.parametrize("n,Hq", [(3, 2), (50, 2), (50, 7)])
def test_values_of_far_apart_magnitudes(gpu, D, bits, n, Hq):
    """Tokens of V far above or below the others: rows that do not see them, other head-dim
    groups and rows that see small ones alone keep their own values' precision."""
    L, window = 700, 100
    table, pages = paged([L], 32)
    k, v0 = rows(891, 1, 1, L, D), rows(892, 1, 1, L, D)
    q = rows(893, 1, Hq, n, D)
    first = L - n - window + 1          # the first key that row 0 sees
    g = torch.Generator().manual_seed(5)
    spread = torch.randint(-40, 40, (L,), generator=g).float().exp2().bfloat16().cuda()
    for what in ("behind", "seen by some", "half a row", "spread"):
        v = v0.clone()
        if what == "behind":
            v[0, 0, first - 1] *= 1e30
        elif what == "seen by some":
            v[0, 0, first + 1] *= 1e30
        elif what == "half a row":
            v[..., :64] *= 2.0 ** -45
            v[..., 70:] *= 2.0 ** 20
        else:
            v *= spread[None, None, :, None]
        cache = fresh_cache(pages, 1, D, 32, bits)
        va.cache_write(cache, k, v, table, int32([L]))
        o, lse = va.cache_attn(q, cache, table, int32([L]), window=window, return_lse=True)
        ref.check(o, lse, ref.cache_attn(q, [k[0].cpu()], [v[0].cpu()], bits, [L], None, window),
                  what)


@pytest.mark.parametrize("D,bits,page", FORMATS)
@pytest.mark.parametrize("n,Hq,H", [(4, 8, 1), (3, 14, 2), (12, 8, 1), (20, 16, 2)])
def test_long_sequences_of_several_tokens(gpu, n, Hq, H, D, bits, page):
    """32, 21, 96 and 160 rows per key/value head over sequences in many chunks."""
    attn_case(895, [6001, 1700, n, 40], Hq, H, n, D, bits, page)
