"""Attention over the cache where the two halves of K's head-dim values have steps of very
different size, down to the smallest that the format holds (2^-100) and 0; bounds in
window_reference."""
import pytest
import torch

import paper_2603_29494_amd as va
import window_reference as ref

pytestmark = pytest.mark.gpu


def rows(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).bfloat16().cuda()


def keys(kind, small, L):
    """K [1, 1, L, 128]: one half N(0, 1) times `small`, the other as named."""
    k = rows(11, 1, 1, L, 128) * small
    half = slice(0, 64) if kind.startswith("first") else slice(64, 128)
    if kind.endswith("zero"):
        k[..., half] = 0
    elif kind.endswith("flat"):
        k[..., half] = small
    else:   # a step near the smallest that is held
        k[..., half] = rows(12, 1, 1, L, 64) * 2.0 ** -98
    return k


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n", [1, 10, 20, 90])   # 2, 20, 40 and 180 rows per key/value head
@pytest.mark.parametrize("kind", ["first zero", "last zero", "first flat", "last flat",
                                  "first small", "last small"])
@pytest.mark.parametrize("small", [2.0 ** -88, 2.0 ** -70, 1.0])
def test_halves_of_different_steps(gpu, small, kind, n, bits):
    """The scores are near 1: q is as large as K's larger half is small."""
    L, D = 200, 128
    k, v, q = keys(kind, small, L), rows(13, 1, 1, L, D), rows(14, 1, 2, n, D) / small
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    cache = va.cache_alloc(4, 1, D, 64, bits)
    cache.data.fill_(0xFF)
    va.cache_write(cache, k, v, table, lens)
    o, lse = va.cache_attn(q, cache, table, lens, return_lse=True)
    ref.check(o, lse, ref.cache_attn(q, [k[0].cpu()], [v[0].cpu()], bits, [L]))
