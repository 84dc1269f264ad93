"""The bounds of sum_bounds on the host: a plain fp32 computation is within them, and planted
mistakes are not."""
import math

import pytest
import torch

import sum_bounds as sb
import window_reference as ref


@pytest.fixture(autouse=True)
def two_threads():
    """Small products: more threads wait for each other, above all beside other test processes."""
    n = torch.get_num_threads()
    torch.set_num_threads(min(n, 2))
    yield
    torch.set_num_threads(n)


def plain32(q, k, v, mask, scale):
    """One head in fp32: lse and o, rounded to bf16."""
    x = ((q.float() @ k.float().t()) * scale).masked_fill(~mask, -math.inf)
    return torch.logsumexp(x, 1), (torch.softmax(x, 1) @ v.float()).bfloat16()


def cache32(q, ks, vs, bits, window, sinks, scale):
    n, out = q.shape[2], []
    for b, L in enumerate(sb.LENS):
        mask = ref.sees(torch.arange(n) + L - n, torch.arange(L), window, sinks, True, L)
        k, v = ref.held(ks[b][0], bits), ref.held(vs[b][0], bits)
        out += [plain32(q[b, h], k, v, mask, scale) for h in range(q.shape[1])]
    return tuple(torch.stack(x).unflatten(0, q.shape[:2]) for x in zip(*out))


def lse_misses(got, want):
    return sb.misses(got[0], want[0], want[1])


def o_misses(got, want):
    return sb.misses(got[-1] if len(got) == 2 else got[2], want[2], want[3])


@pytest.mark.parametrize("n,Hq", sb.ROWS)
@pytest.mark.parametrize("D,bits", [(64, 4), (64, 8), (128, 4), (128, 8)])
@pytest.mark.parametrize("which", sb.SCALES)
def test_cache_bounds(which, D, bits, n, Hq):
    q, ks, vs, scale = sb.cache_case(n, Hq, D, which)
    for window, sinks in sb.WINDOWS:
        window = window or 1 << 30
        want = sb.cache_attn(q, ks, vs, bits, sb.LENS, window, sinks, scale)
        got = cache32(q, ks, vs, bits, window, sinks, scale)
        assert lse_misses(got, want) <= 1 and o_misses(got, want) <= 1

        def wrong(w=window, s=sinks, **mistake):
            return sb.cache_attn(q, ks, vs, bits, sb.LENS, w, s, scale, **mistake)
        if which == "few keys":     # keys held in fewer bits
            for t in (torch.bfloat16, torch.float16):
                assert lse_misses(wrong(k_as=t), want) > 1, t
        else:
            assert o_misses(wrong(v_mask=254), want) > 1     # V's codes a bit short
            for w, s in ((window + 1, sinks), (window - 1, sinks), (window, sinks + 1),
                         (window, sinks - 1)):               # a key too many or too few
                if sinks:
                    assert lse_misses(wrong(w, s), want) > 1, (w, s)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_window_bounds(causal, D):
    for which in sb.SCALES:
        q, k, v, scale = sb.window_case(D, which)

        def form(k, w=300, s=20):
            return sb.window_attn(q, k, v, w, s, causal, scale)
        want = form(k)
        mask = ref.sees(torch.arange(700), torch.arange(700), 300, 20, causal, 700)
        got = [plain32(q[b, h], k[b, 0], v[b, 0], mask, scale) for b in range(2) for h in range(2)]
        got = tuple(torch.stack(x).unflatten(0, (2, 2)) for x in zip(*got))
        assert lse_misses(got, want) <= 1 and o_misses(got, want) <= 1
        if which == "many keys":
            for w, s in ((301, 20), (299, 20), (300, 21), (300, 19)):
                assert lse_misses(form(k, w, s), want) > 1, (w, s)
        else:    # scores off by an eighth of an fp16 step
            assert lse_misses(form(k.double() * (1 + 2.0 ** -14)), want) > 1
