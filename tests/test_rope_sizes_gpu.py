"""Rotary positions of sizes that change how the work is dealt out: heads walked over by a wave,
tensors past the caches, more tokens than one dimension of a launch holds."""
import pytest
import torch

import paper_2603_29494_amd as va
from test_rope_gpu import check

pytestmark = pytest.mark.gpu


def test_more_tokens_than_a_launch_dimension_holds(gpu):
    """2^26 single tokens, a quarter of a workgroup each: 2^32 threads and some."""
    B = (1 << 26) + 5
    plan = va.rope_plan(64, layout="half")
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.empty(B, 1, 1, 64, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    pos = (torch.arange(B, dtype=torch.int32, device="cuda") % 100003).view(1, B, 1)
    y = va.rope(plan, q, pos=pos)
    torch.cuda.synchronize()
    half = B // 2   # as two calls give it
    for a, b in ((0, half), (half, B)):
        same = torch.equal(y[a:b], va.rope(plan, q[a:b], pos=pos[:, a:b]))
        assert same, (a, b)
    for a in (0, half, B - 300):
        check(plan, q[a:a + 300], y[a:a + 300], pos[:, a:a + 300])


def normal(seed, B, H, N, D, head_major):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (B, H, N, D) if head_major else (B, N, H, D)
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    return x if head_major else x.transpose(1, 2)


def bits(x):
    return x.contiguous().view(torch.int16)


def against_slices(plan, q, k, step, **kw):
    """The whole call against calls of `step` tokens at a time, bit for bit, and tokens from all over
    it against 64 bits; then in place."""
    B, _, N, _ = q.shape
    g = torch.Generator().manual_seed(N)
    pos = torch.randint(0, 200000, (plan.axes, B, N), generator=g).int().cuda()
    yq, yk = va.rope(plan, q, k, pos=pos, **kw)
    torch.cuda.synchronize()
    for a in range(0, N, step):
        z = slice(a, min(N, a + step))
        pq, pk = va.rope(plan, q[:, :, z], k[:, :, z], pos=pos[:, :, z], **kw)
        for x, y in ((pq, yq[:, :, z]), (pk, yk[:, :, z])):
            assert torch.equal(bits(x), bits(y)), a
    at = torch.randperm(N, generator=g)[:40].sort()[0].cuda()
    for x, y in ((q, yq), (k, yk)):
        check(plan, x[:, :, at], y[:, :, at], pos[:, :, at], kw.get("transpose", False))
    va.rope(plan, q, k, pos=pos, out=(q, k), **kw)
    assert torch.equal(bits(q), bits(yq)) and torch.equal(bits(k), bits(yk))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,D", [(128, 128), (100, 128), (64, 64), (18, 64)])
@pytest.mark.parametrize("head_major", [True, False])
def test_several_heads_per_wave_and_turn(gpu, layout, rot, D, head_major):
    """Tokens enough that a wave walks over heads with the same angles, 32 MB in and out."""
    plan = va.rope_plan(rot, layout=layout, sections=(1, rot // 2 - 1))
    N = 1700 if D == 128 else 3000
    q, k = (normal(s, 2, H, N, D, head_major) for s, H in ((1, 40), (2, 9)))
    against_slices(plan, q, k, 97)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,D", [(128, 128), (100, 128), (64, 64), (18, 64)])
@pytest.mark.parametrize("head_major", [True, False])
def test_tensors_past_the_caches(gpu, layout, rot, D, head_major):
    """More than 256 MB in and out, which go past the caches; calls of half the tokens do not."""
    plan = va.rope_plan(rot, layout=layout)
    N = 14001 if D == 128 else 28001
    q, k = (normal(s, 1, H, N, D, head_major) for s, H in ((3, 32), (4, 8)))
    assert 4 * N * 40 * D > 1 << 28 > 4 * (N // 2 + 1) * 40 * D
    against_slices(plan, q, k, N // 2 + 1, transpose=D == 64)


def test_padding_past_the_caches(gpu):
    """Rows that do not exist are 0 in an output made here, and stay in a given one."""
    plan = va.rope_plan(128, layout="half")
    N = 7100
    q, k = normal(5, 2, 32, N, 128, False), normal(6, 2, 8, N, 128, True)
    lens, n_new = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([9000, 7], [N, 5]))
    yq, yk = va.rope(plan, q, k, lens=lens, n_new=n_new)
    out = (torch.full_like(q, 3.0), torch.full_like(k, 3.0))
    va.rope(plan, q, k, lens=lens, n_new=n_new, out=out)
    for x, y, z in ((q, yq, out[0]), (k, yk, out[1])):
        assert (y[1, :, 5:] == 0).all() and (z[1, :, 5:] == 3.0).all()
        assert torch.equal(bits(y[0]), bits(z[0])) and torch.equal(bits(y[1, :, :5]), bits(z[1, :, :5]))
        for b, n, first in ((0, N, 9000 - N), (1, 5, 2)):
            at = torch.arange(0, n, max(1, n // 17))
            check(plan, x[b:b + 1, :, at], y[b:b + 1, :, at], (first + at)[None, None])
