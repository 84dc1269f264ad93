"""Window attention where scores jump within a row and V is large, so that a weight taken against
the row's first keys, times V, is past fp32; bounds in window_reference."""
import math

import pytest
import torch

import paper_2603_29494_amd as va
import window_reference as ref

pytestmark = pytest.mark.gpu


def rows(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).bfloat16().cuda()


def jumping(N, D, jump, at):
    """q, k [1, 1, N, D]: scores near 0 for keys before `at`, near `jump` from it on."""
    q, k = rows(1, 1, 1, N, D) / 8, rows(2, 1, 1, N, D) / 8
    q[..., 0] = 8.0
    k[..., 0] = 0
    k[:, :, at:, 0] = jump / 8 * math.sqrt(D)
    return q, k


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("at", [64, 130])
@pytest.mark.parametrize("jump,size", [(40, 2.0 ** 67), (63, 2.0 ** 34), (68, 2.0 ** 34),
                                       (86, 2.0 ** 20), (95, 1.0), (20, 2.0 ** 97),
                                       (300, 2.0 ** 97)])
def test_a_jump_of_the_scores_under_large_values(gpu, jump, size, at, causal, D):
    """From just below what the weights' sum can hold to far past it."""
    N = 300
    q, k = jumping(N, D, jump, at)
    v = rows(3, 1, 1, N, D) * size
    o, lse = va.window_attn(q, k, v, 250, 3, causal, return_lse=True)
    ref.check(o, lse, ref.window_attn(q, k, v, 250, 3, causal), f"{jump} {size}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("jump", [5, 20, 60, 80])
def test_a_hidden_key_changes_no_bit_where_scores_jump(gpu, jump, D):
    """The rows that do not see a NaN of V come out as without it, however their references
    move."""
    N, window, nan = 400, 150, 40
    q, k = jumping(N, D, jump, 130)
    v = rows(3, 1, 1, N, D)
    clean = va.window_attn(q, k, v, window, 0, True)
    v[:, :, nan, 5] = math.nan
    o = va.window_attn(q, k, v, window, 0, True)
    hidden = ~ref.sees(torch.arange(N), torch.arange(N), window, 0, True, N)[:, nan].cuda()
    assert torch.equal(o[:, :, hidden], clean[:, :, hidden])
    assert o[:, :, ~hidden][..., 5].isnan().all()
