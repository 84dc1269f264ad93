"""Rotary positions against a plain 64-bit form.

Bound.  With c = f cos t, s = f sin t of the kernel: the reduced angle is off by a relative 2^-23
(its rounding to fp32 and the product with pi / 2), the polynomial by four roundings, the factor by
one, so c and s by at most f (2^-22 + 2^-24); each of two products and their sum round once more, 2^-24
each.  Together (|a| + |b|) f 2^-21 is above it.  The frequency as turns is off by 2^-51 of it, which
a far position multiplies: (|a| + |b|) f |t| 2^-51.  The result is rounded once, 2^-8 of it."""
import math

import pytest
import torch

import paper_2603_29494_amd as va

pytestmark = pytest.mark.gpu


def rows(seed, B, H, N, D, head_major=True):
    g = torch.Generator().manual_seed(seed)
    if head_major:
        return torch.randn(B, H, N, D, generator=g).bfloat16().cuda()
    return torch.randn(B, N, H, D, generator=g).bfloat16().cuda().transpose(1, 2)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def turned(plan, x, pos, transpose=False):
    """x [B, H, N, D] turned by pos [axes, B, N] in 64 bits, and its bound."""
    x, pos = x.cpu().double(), pos.cpu().double()
    n = len(plan.freq)
    freq = torch.tensor(plan.freq, dtype=torch.float64)
    t = pos[torch.tensor(plan.axis)].permute(1, 2, 0) * freq        # [B, N, pairs]
    t = (-t if transpose else t)[:, None]
    at = torch.arange(n)
    ia, ib = (at, at + n) if plan.layout == "half" else (2 * at, 2 * at + 1)
    a, b = x[..., ia], x[..., ib]
    y, e = x.clone(), torch.zeros_like(x)
    y[..., ia] = plan.factor * (a * torch.cos(t) - b * torch.sin(t))
    y[..., ib] = plan.factor * (a * torch.sin(t) + b * torch.cos(t))
    # the reference's own angle is off by 2^-53 of it as well
    e[..., ia] = e[..., ib] = (a.abs() + b.abs()) * abs(plan.factor) * (2.0 ** -21 + t.abs() * 2.0 ** -50)
    return y, e + 2.0 ** -8 * y.abs() * (e > 0) + 2.0 ** -133 * (e > 0)


def check(plan, x, y, pos, transpose=False, label=""):
    ref, bound = turned(plan, x, pos, transpose)
    over = ((y.cpu().double() - ref).abs() - bound).max()
    assert over <= 0, f"{label}: past its bound by {over:.3e}"


def grid(axes, B, N, start=0):
    return (start + torch.arange(N)).expand(axes, B, N)


PLANS = [dict(rot=128, D=128), dict(rot=64, D=128), dict(rot=48, D=64), dict(rot=20, D=64),
         dict(rot=2, D=64), dict(rot=126, D=128), dict(rot=96, D=128, sections=(16, 20, 12)),
         dict(rot=64, D=64, sections=(10, 11, 11), own_ladders=True)]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("p", PLANS, ids=lambda p: f"{p['rot']}of{p['D']}")
@pytest.mark.parametrize("head_major", [True, False])
def test_against_the_formula(gpu, p, layout, head_major):
    p = dict(p)
    D = p.pop("D")
    plan = va.rope_plan(layout=layout, **p)
    for B, Hq, Hk, N in ((1, 1, 1, 1), (2, 5, 3, 37), (1, 7, 1, 130), (3, 40, 8, 2)):
        q, k = rows(B, B, Hq, N, D, head_major), rows(B + 9, B, Hk, N, D, head_major)
        pos = torch.randint(-50, 200000, (plan.axes, B, N),
                            generator=torch.Generator().manual_seed(N)).int()
        yq, yk = va.rope(plan, q, k, pos=pos.cuda())
        torch.cuda.synchronize()
        check(plan, q, yq, pos, label="q")
        check(plan, k, yk, pos, label="k")
        # transposed, and q alone
        back = va.rope(plan, q, pos=pos.cuda(), transpose=True)
        check(plan, q, back, pos, True, "transposed")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_where_positions_come_from(gpu, layout):
    plan = va.rope_plan(128, layout=layout, sections=(20, 22, 22))
    B, N = 3, 50
    q, k = rows(1, B, 4, N, 128, False), rows(2, B, 2, N, 128)
    yq, yk = va.rope(plan, q, k, start=-7)
    check(plan, q, yq, grid(3, B, N, -7))
    check(plan, k, yk, grid(3, B, N, -7))
    # the last rows of sequences, padded; padded rows of a given output are left as they were
    lens, n_new = [60, 3, 4000], [50, 9, 0]
    out = (torch.full_like(q, 5.0), torch.full_like(k, 5.0))
    zq, zk = va.rope(plan, q, k, lens=int32(lens), n_new=int32(n_new), out=out)
    assert zq is out[0] and zk is out[1]
    for b in range(B):
        n = n_new[b]
        pos = grid(3, 1, n, lens[b] - n)
        for x, z in ((q, zq), (k, zk)):
            if n:
                check(plan, x[b:b + 1, :, :n], z[b:b + 1, :, :n], pos)
            assert (z[b, :, n:] == 5.0).all()
    yq, yk = va.rope(plan, q, k, lens=int32(lens))
    for b in range(B):
        check(plan, q[b:b + 1], yq[b:b + 1], grid(3, 1, N, lens[b] - N))
    # n_new out of range is clamped, and padding of an output made here is 0
    yq = va.rope(plan, q, lens=int32(lens), n_new=int32([99, -4, 1]))
    check(plan, q[:1], yq[:1], grid(3, 1, N, 60 - N))
    assert (yq[1] == 0).all() and (yq[2, :, 1:] == 0).all()
    # positions shared by the sequences, and with n_new
    pos = torch.randint(0, 9999, (3, 1, N)).int().cuda().expand(3, B, N)
    yq = va.rope(plan, q, pos=pos, n_new=int32([N, 20, N]))
    check(plan, q[::2], yq[::2], pos[:, ::2])
    assert (yq[1, :, 20:] == 0).all()


def test_far_positions(gpu):
    """Angles of a billion radians: reduced before they are rounded."""
    plan = va.rope_plan(64, base=500000.0, layout="half")
    q = rows(3, 1, 2, 40, 64)
    pos = torch.cat([torch.arange(10), 131072 + torch.arange(10), 2 ** 30 - torch.arange(10),
                     -2 ** 31 + torch.arange(10)])[None, None].int()
    check(plan, q, va.rope(plan, q, pos=pos.cuda()), pos)
    check(plan, q, va.rope(plan, q, start=2 ** 30), grid(1, 1, 40, 2 ** 30))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,D", [(128, 128), (32, 128), (20, 64), (50, 64)])
def test_in_place_and_what_is_not_turned(gpu, layout, rot, D):
    plan = va.rope_plan(rot, layout=layout)
    for head_major in (True, False):
        q, k = rows(4, 2, 6, 33, D, head_major), rows(5, 2, 3, 33, D, head_major)
        if rot < D:   # bits behind the turned values, NaN and infinities among them
            q[..., rot], q[..., D - 1], k[..., rot] = math.nan, math.inf, -0.0
        yq, yk = va.rope(plan, q, k, start=3)
        for x, y in ((q, yq), (k, yk)):
            assert torch.equal(x.view(torch.int16)[..., rot:], y.view(torch.int16)[..., rot:])
        q2, k2 = q.clone(), k.clone()
        va.rope(plan, q2, k2, start=3, out=(q2, k2))
        assert torch.equal(q2.view(torch.int16), yq.view(torch.int16))
        assert torch.equal(k2.view(torch.int16), yk.view(torch.int16))
        # only one of them in place
        q3, k3 = q.clone(), torch.zeros_like(k)
        va.rope(plan, q3, k, start=3, out=(q3, k3))
        assert torch.equal(q3.view(torch.int16), yq.view(torch.int16))
        assert torch.equal(k3.view(torch.int16), yk.view(torch.int16))


def test_gradient_is_the_transposed_turn(gpu):
    """<dy, R x> = <R' dy, x> for the formula's R (its matrix transposed), and against differences:
    the turn is linear, so a difference of any size is its derivative."""
    for scaling in (None, "parts"):
        plan = va.rope_plan(64, layout="interleaved", scaling=scaling, factor=8.0, context=4096)
        x, dy, d = rows(6, 1, 2, 19, 64), rows(7, 1, 2, 19, 64), rows(8, 1, 2, 19, 64)
        dx = va.rope(plan, dy, start=11, transpose=True).double()
        # derivative of <dy, R x> along d: two calls whose inputs differ by d
        hi = (x.float() + d.float()).bfloat16()
        step = hi.double() - x.double()
        diff = (dy.double() * (va.rope(plan, hi, start=11).double()
                               - va.rope(plan, x, start=11).double())).sum()
        want = (dx * step).sum()
        # every value of the two turns and of dx is off by 2^-8 of it at most (and fp32)
        scale = plan.factor * 2 ** -8 * 1.01
        slack = (dy.double().abs() * scale * 1.5 * (hi.double().abs() + x.double().abs()
                                                    + _partner(hi) + _partner(x))).sum() \
            + (scale * 1.5 * (dy.double().abs() + _partner(dy)) * step.abs()).sum()
        assert (diff - want).abs() <= slack
        pos = grid(1, 1, 19, 11)
        check(plan, dy, va.rope(plan, dy, start=11, transpose=True), pos, True)


def _partner(x):
    return x.double().abs().unflatten(-1, (-1, 2)).flip(-1).flatten(-2)


def test_strides_and_shared_heads(gpu):
    """Slices of a packed projection, a head that all sequences share, other strides for outputs."""
    plan = va.rope_plan(128, layout="half")
    packed = rows(9, 2, 12, 45, 128, False).transpose(1, 2).contiguous()   # [B, N, 12, D]
    q, k = packed[:, :, :8].transpose(1, 2), packed[:, :, 8:10].transpose(1, 2)
    out = (torch.zeros(2, 8, 45, 128, dtype=torch.bfloat16, device="cuda"),
           torch.zeros(2, 45, 2, 128, dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    va.rope(plan, q, k, start=5, out=out)
    check(plan, q, out[0], grid(1, 2, 45, 5))
    check(plan, k, out[1], grid(1, 2, 45, 5))
    one = rows(10, 1, 1, 45, 128).expand(2, 4, 45, 128)
    check(plan, one, va.rope(plan, one, start=2), grid(1, 2, 45, 2))
    # in place within the packed tensor: the rest of it stays
    before = packed.clone()
    va.rope(plan, q, k, start=5, out=(q, k))
    assert torch.equal(packed[:, :, 10:], before[:, :, 10:])
    assert torch.equal(q, out[0]) and torch.equal(k, out[1])


def test_stream_and_replayed_graph(gpu):
    plan = va.rope_plan(128, layout="interleaved")
    q, k = rows(11, 2, 4, 1, 128), rows(12, 2, 2, 1, 128)
    lens = int32([5, 900])
    out = (torch.zeros_like(q), torch.zeros_like(k))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        va.rope(plan, q, k, lens=lens, out=out)
    side.synchronize()
    check(plan, q, out[0], torch.tensor([[[4], [899]]]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        va.rope(plan, q, k, lens=lens, out=out)
    for i in range(4):
        lens.add_(1)
        q.copy_(rows(20 + i, 2, 4, 1, 128))
        graph.replay()
        torch.cuda.synchronize()
        check(plan, q, out[0], torch.tensor([[[5 + i], [900 + i]]]))
        assert torch.equal(out[0], va.rope(plan, q, lens=lens))
