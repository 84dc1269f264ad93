"""Attention over another sequence's keys against a plain 64-bit form; bounds in window_reference
(weights rounded to bf16, sums in fp32)."""
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


def cross64(q, k, v, lens=None, mask=None, n_q=None, scale=0.0):
    """All heads; rows that do not exist are NaN.  Masked and absent keys are taken out first."""
    q, k, v = (t.cpu().double() for t in (q, k, v))
    B, Hq, Nq, D = q.shape
    Hkv, Nk = k.shape[1:3]
    scale = scale or D ** -0.5
    o, ob = torch.full_like(q, math.nan), torch.zeros_like(q)
    lse = torch.full((B, Hq, Nq), math.nan, dtype=torch.float64)
    lb = torch.zeros_like(lse)
    for b in range(B):
        L = Nk if lens is None else min(max(int(lens[b]), 0), Nk)
        n = Nq if n_q is None else min(max(int(n_q[b]), 0), Nq)
        at = torch.arange(L)
        if mask is not None:
            at = at[mask[b, :L].cpu().bool()]
        see = torch.ones(n, len(at), dtype=torch.bool)
        for h in range(Hq):
            g = h // (Hq // Hkv)
            if n == 0:
                continue
            if len(at) == 0:
                o[b, h, :n], lse[b, h, :n] = 0.0, -math.inf
                continue
            o[b, h, :n], lse[b, h, :n], ob[b, h, :n], lb[b, h, :n] = ref.attend(
                q[b, h, :n], k[b, g][at], v[b, g][at], see, scale)
    return o, lse, ob, lb


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (6, 2), (7, 1)])
@pytest.mark.parametrize("Nq,Nk", [(1, 1), (1, 33), (2, 700), (5, 31), (4, 2500), (11, 64), (33, 1),
                                   (40, 65), (129, 128), (300, 77), (70, 1500), (1, 9000)])
def test_against_the_formula(gpu, D, Hq, Hkv, Nq, Nk):
    B = 2 if Nk < 3000 else 1
    q, k, v = rows(1, B, Hq, Nq, D), rows(2, B, Hkv, Nk, D), rows(3, B, Hkv, Nk, D)
    k[:, :, 0] += 2 * q[:, :Hkv, 0]     # a key that stands out
    o, lse = va.cross_attn(q, k, v, return_lse=True)
    torch.cuda.synchronize()
    ref.check(o, lse, cross64(q, k, v))


@pytest.mark.parametrize("D,H,Nq,Nk", [(64, 9, 37, 3500), (128, 9, 37, 3500), (64, 17, 33, 6600)])
def test_many_row_tiles_over_many_keys(gpu, D, H, Nq, Nk):
    """More row tiles than half of the CUs, and than all, and keys enough to be cut, some lengths
    within the first piece."""
    B = 16
    q, k, v = rows(21, B, H, Nq, D), rows(22, B, H, Nk, D), rows(23, B, H, Nk, D)
    lens = [Nk, 0, 1, Nk - 1, 1167, 1280, 1281, 2560, 2561, 3000] + [Nk] * 6
    o, lse = va.cross_attn(q, k, v, lens=int32(lens), return_lse=True)
    ref.check(o, lse, cross64(q, k, v, lens=lens))


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 4), (128, 6, 2)])
@pytest.mark.parametrize("Nq", [1, 7, 50, 200])
@pytest.mark.parametrize("Nk", [45, 700, 2100])
def test_lengths_masks_and_padding(gpu, D, Hq, Hkv, Nq, Nk):
    """Sequences of no keys, of one, of all; rows of a mask that leave nothing, and half; what is
    hidden is NaN and infinite, and padded rows stay."""
    B = 6
    lens, n_q = [0, 1, Nk, Nk + 9, Nk // 2 + 1, Nk - 1], [Nq, Nq, Nq, 0, max(1, Nq // 2), Nq + 3]
    q, k, v = rows(4, B, Hq, Nq, D), rows(5, B, Hkv, Nk, D), rows(6, B, Hkv, Nk, D)
    mask = torch.rand(B, Nk, generator=torch.Generator().manual_seed(Nk)) < 0.5
    mask[5] = False
    mask[2, :Nk // 2] = False           # whole tiles of nothing first
    for b in range(B):
        L = min(lens[b], Nk)
        gone = ~mask[b]
        gone[L:] = True
        gone = gone.cuda()
        k[b, :, gone], v[b, :, gone] = math.nan, math.inf
    out = torch.full_like(q, 9.0)
    for m in (mask.cuda(), mask.to(torch.uint8).cuda() * 255):
        o, lse = va.cross_attn(q, k, v, lens=int32(lens), mask=m, n_q=int32(n_q), out=out,
                               return_lse=True)
        torch.cuda.synchronize()
        ref.check(o, lse, cross64(q, k, v, lens, mask, n_q))
        for b in range(B):
            n = min(n_q[b], Nq)
            assert (o[b, :, n:] == 9.0).all() and (lse[b, :, n:] == 0).all()
    # an output made by the call: its padding is 0
    o, lse = va.cross_attn(q, k, v, lens=int32(lens), mask=mask.cuda(), n_q=int32(n_q),
                           return_lse=True)
    ref.check(o, lse, cross64(q, k, v, lens, mask, n_q))
    for b in range(B):
        n = min(n_q[b], Nq)
        assert (o[b, :, n:] == 0).all() and (lse[b, :, n:] == 0).all()
    # lengths alone: only what is past them hides
    for b in range(B):
        k[b, :, :min(lens[b], Nk)], v[b, :, :min(lens[b], Nk)] = (
            rows(7 + b, Hkv, min(lens[b], Nk), D), rows(17 + b, Hkv, min(lens[b], Nk), D))
    o, lse = va.cross_attn(q, k, v, lens=int32(lens), return_lse=True)
    ref.check(o, lse, cross64(q, k, v, lens))


def test_many_sequences_and_uneven_lengths(gpu):
    """More sequences than are dealt out by their lengths, and as many with lengths far apart."""
    for B, Nk in ((300, 600), (256, 1100), (33, 3000), (256, 4200), (130, 5000)):
        q, k, v = rows(1, B, 2, 1, 64), rows(2, B, 1, Nk, 64), rows(3, B, 1, Nk, 64)
        lens = (torch.rand(B, generator=torch.Generator().manual_seed(B)) ** 4 * (Nk + 1)).int()
        lens[0], lens[-1] = Nk, 0
        o, lse = va.cross_attn(q, k, v, lens=lens.cuda(), return_lse=True)
        ref.check(o, lse, cross64(q, k, v, lens=lens.tolist()))


@pytest.mark.parametrize("Nq", [1, 90])
def test_large_values_and_scales(gpu, Nq):
    """Scores that jump past fp32's exponentials late in the walk, tiny ones, and a scale of 0 and
    nearly 0."""
    D, Nk = 128, 800
    q, v = rows(1, 1, 2, Nq, D, scale=4.0), rows(3, 1, 2, Nk, D, scale=1e3)
    k = rows(2, 1, 2, Nk, D) * torch.linspace(0.01, 60, Nk).cuda()[None, None, :, None]
    k = k.bfloat16()
    k[:, :, 700] = 30 * q[:, :, 0]
    for scale in (0.0, 1.0, 1e-3, 1e-38):
        o, lse = va.cross_attn(q, k, v, scale=scale, return_lse=True)
        ref.check(o, lse, cross64(q, k, v, scale=scale))
    mask = torch.arange(Nk).cuda()[None] % 3 > 0
    o, lse = va.cross_attn(q, k, v, scale=1e-38, mask=mask, return_lse=True)
    ref.check(o, lse, cross64(q, k, v, mask=mask, scale=1e-38))


def test_nan_in_a_visible_key_and_in_a_row(gpu):
    """A NaN row of q is its own row's; a NaN value of V is that value of every row."""
    for Nq in (3, 60):
        q, k, v = rows(1, 1, 2, Nq, 64), rows(2, 1, 1, 300, 64), rows(3, 1, 1, 300, 64)
        clean = va.cross_attn(q, k, v)
        q[0, 1, 2, 5] = math.nan
        o = va.cross_attn(q, k, v)
        assert o[0, 1, 2].isnan().all()
        keep = torch.ones(2, Nq, dtype=torch.bool)
        keep[1, 2] = False
        assert torch.equal(o[0][keep], clean[0][keep])
        v[0, 0, 200, 7] = math.nan
        o = va.cross_attn(q, k, v)
        assert o[0, :, :, 7].isnan().all()
        rest = [d for d in range(64) if d != 7]
        assert torch.equal(o[0][keep][:, rest], clean[0][keep][:, rest])


def test_strides_shared_keys_and_masks(gpu):
    """Token-major rows, one encoder output for all sequences, a mask that all share."""
    D, Nq, Nk = 128, 150, 210
    q = rows(1, 3, Nq, 4, D).transpose(1, 2)
    kv = rows(2, 1, Nk, 2, 2, D)                  # a packed projection of one prompt
    k, v = (kv[:, :, i].transpose(1, 2).expand(3, 2, Nk, D) for i in range(2))
    mask = (torch.arange(Nk) % 5 > 0).cuda()[None].expand(3, Nk)
    out = torch.zeros(3, Nq, 4, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    o, lse = va.cross_attn(q, k, v, mask=mask, out=out, return_lse=True)
    assert o is out
    ref.check(o, lse, cross64(q, k, v, mask=mask))
    # positions of a long buffer past 32 bits of bytes between sequences are strides too
    big = torch.zeros(2, (1 << 30) + 64, dtype=torch.bfloat16, device="cuda")
    qb = big[:, :2 * 5 * 64].view(2, 2, 5, 64)
    qb.copy_(rows(5, 2, 2, 5, 64))
    k2 = rows(6, 2, 2, 40, 64)
    o, lse = va.cross_attn(qb, k2, k2, return_lse=True)
    ref.check(o, lse, cross64(qb, k2, k2))


def test_streams_workspaces_and_a_replayed_graph(gpu):
    """Calls at once, each with a workspace of its own; a captured call follows lens, mask, n_q."""
    D, Nq, Nk, B = 64, 2, 4000, 2
    q, k, v = rows(1, B, 6, Nq, D), rows(2, B, 2, Nk, D), rows(3, B, 2, Nk, D)
    need = va.cross_attn_workspace_bytes(q, k)
    assert need > 0
    alone = va.cross_attn(q, k, v)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(va.cross_attn(q, k, v))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, alone)
    lens, n_q = int32([4000, 3]), int32([2, 1])
    mask = torch.ones(B, Nk, dtype=torch.bool, device="cuda")
    ws, graphs = torch.empty(need, dtype=torch.uint8, device="cuda"), []
    outs = [torch.zeros_like(q) for _ in range(2)]
    qs = [q, rows(9, B, 6, Nq, D)]
    for i in range(2):    # two graphs that share a workspace, replayed one after the other
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            va.cross_attn(qs[i], k, v, lens=lens, mask=mask, n_q=n_q, out=outs[i], workspace=ws)
    for step, (a, b, m) in enumerate(((4000, 3, 1.0), (1, 4000, 0.5), (0, 700, 0.0), (2500, 2500, 0.9))):
        lens.copy_(int32([a, b]))
        mask.copy_(torch.rand(B, Nk, generator=torch.Generator().manual_seed(step)).cuda() < m)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        for i in (step % 2, 1 - step % 2):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            want = va.cross_attn(qs[i], k, v, lens=lens, mask=mask, n_q=n_q)
            assert torch.equal(outs[i][0], want[0]) and torch.equal(outs[i][1, :, :1], want[1, :, :1])
