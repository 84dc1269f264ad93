"""Cross attention of few rows with the bounds of weights held in two bf16 numbers."""
import pytest
import torch

import cross_weights as cw
import paper_2603_29494_amd as va
import window_reference as ref
from test_cross_gpu import cross64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (14, 2)])
@pytest.mark.parametrize("Nq", [1, 2])
@pytest.mark.parametrize("Nk", [2, 5, 33, 257, 700, 9000])
def test_weights_of_few_rows(gpu, D, Hq, Hkv, Nq, Nk):
    """Keys of one tile, of several per wave, and cut into chunks."""
    q, k, v = (x.cuda() for x in cw.inputs(Nk + Nq, 2, Hq, Hkv, Nq, Nk, D))
    o, lse = va.cross_attn(q, k, v, return_lse=True)
    ref.check(o, lse, cw.cross64(q, k, v))
    mask = torch.rand(2, Nk, generator=torch.Generator().manual_seed(Nk)) < 0.5
    mask[:, Nk // 2] = True
    o, lse = va.cross_attn(q, k, v, mask=mask.cuda(), return_lse=True)
    ref.check(o, lse, cw.cross64(q, k, v, mask))


@pytest.mark.parametrize("D", [64, 128])
def test_weights_after_a_jump(gpu, D):
    """References that move within the walk: scores that grow along the keys."""
    q, k, v = (x.cuda() for x in cw.inputs(3, 1, 4, 2, 3, 1500, D))
    k = (k * torch.linspace(0.1, 6, 1500).cuda()[None, None, :, None]).bfloat16()
    o, lse = va.cross_attn(q, k, v, return_lse=True)
    ref.check(o, lse, cw.cross64(q, k, v))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Nq", [1, 5, 9, 60])
@pytest.mark.parametrize("Nk", [40, 3000])
def test_infinities_in_visible_keys(gpu, D, Nq, Nk):
    """An infinity of V that a row weighs is one of its result, of either sign; the other values are
    what they are without it."""
    q, k, v = (x.cuda() for x in cw.inputs(4, 1, 4, 2, Nq, Nk, D))
    q = q / 8
    clean = va.cross_attn(q, k, v)
    v[:, :, Nk // 3, 5], v[:, :, Nk - 1, 20] = float("inf"), float("-inf")
    o = va.cross_attn(q, k, v)
    assert (o[..., 5] == float("inf")).all() and (o[..., 20] == float("-inf")).all()
    rest = [d for d in range(D) if d not in (5, 20)]
    assert torch.equal(o[..., rest], clean[..., rest])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Nq", [1, 9, 60])
def test_jumping_scores_under_large_values(gpu, D, Nq):
    """V near 2^90, the largest that is promised, and scores that jump by up to 300 along the keys."""
    q, k, v = (x.cuda() for x in cw.inputs(5, 1, 2, 1, Nq, 900, D))
    k = (k * torch.linspace(0.1, 40, 900).cuda()[None, None, :, None]).bfloat16()
    k[:, :, 700] = 8 * q[:, :1, 0]
    v = (v.clamp(-3.9, 3.9) * 2.0 ** 88).bfloat16()
    o, lse = va.cross_attn(q, k, v, return_lse=True)
    ref.check(o, lse, cw.cross64(q, k, v) if 2 * Nq <= 16 else cross64(q, k, v))
