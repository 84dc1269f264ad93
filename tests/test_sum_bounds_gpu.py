"""Window attention and attention over the cache: outputs off by no more than the kernels' roundings
of weights and values add up to, log-sum-exps by no more than fp32 sums (sum_bounds)."""
import pytest
import torch

import paper_2603_29494_amd as va
import sum_bounds as sb

pytestmark = pytest.mark.gpu


def check(label, o, lse, want):
    r = sb.misses(lse, want[0], want[1]), sb.misses(o, want[2], want[3])
    rms = (lse.cpu().double() - want[0]).square().mean().sqrt()
    print(f"{label}: lse {r[0]:.3f} (rms {rms:.1e}), o {r[1]:.3f}")
    assert max(r) <= 1, label


@pytest.mark.parametrize("n,Hq", sb.ROWS)
@pytest.mark.parametrize("D,bits", [(64, 4), (64, 8), (128, 4), (128, 8)])
@pytest.mark.parametrize("which", sb.SCALES)
def test_cache_attn(gpu, which, D, bits, n, Hq):
    q, ks, vs, scale = sb.cache_case(n, Hq, D, which)
    cols = -(-max(sb.LENS) // 64)
    table = torch.arange(len(ks) * cols, dtype=torch.int32, device="cuda").view(len(ks), cols)
    lens = torch.tensor(sb.LENS, dtype=torch.int32, device="cuda")
    cache = va.cache_alloc(len(ks) * cols, 1, D, 64, bits)
    for b, (k, v) in enumerate(zip(ks, vs)):
        va.cache_write(cache, k[None].cuda(), v[None].cuda(), table[b:b + 1], lens[b:b + 1])
    for window, sinks in sb.WINDOWS:
        o, lse = va.cache_attn(q.cuda(), cache, table, lens, window=window, sinks=sinks,
                               scale=scale, return_lse=True)
        check(f"{which} D={D} {bits} bits {n}x{Hq} window {window}", o, lse,
              sb.cache_attn(q, ks, vs, bits, sb.LENS, window or 1 << 30, sinks, scale))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("which", sb.SCALES)
def test_window_attn(gpu, which, causal, D):
    q, k, v, scale = sb.window_case(D, which)
    o, lse = va.window_attn(q.cuda(), k.cuda(), v.cuda(), 300, 20, causal, scale=scale,
                            return_lse=True)
    check(f"{which} D={D} causal={causal}", o, lse,
          sb.window_attn(q, k, v, 300, 20, causal, scale))
