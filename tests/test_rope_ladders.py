"""Ladders of frequencies whose slow end lies past the last pair: the last pair makes more than
`slow` turns over the context, so no pair is divided in full."""
import math

import pytest

import paper_2603_29494_amd as va


def shares(rot, base, context, factor, fast, slow):
    """Share of f_i / factor in pair i's frequency, from the definition: 0 up to the pair that makes
    `fast` turns over the context, 1 from the one that makes `slow` on, linear in i between, both
    rounded outwards, the first no lower than 0, the second no higher than rot - 1."""
    half = rot // 2

    def pair(turns):   # base^(-i / half) context = 2 pi turns
        return half * (math.log(context) - math.log(2 * math.pi * turns)) / math.log(base)
    first, last = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot - 1)
    return [0.0 if i <= first else 1.0 if i >= last else (i - first) / (last - first)
            for i in range(half)]


@pytest.mark.parametrize("rot,base,context", [
    (128, 1e4, 131072), (128, 1e4, 65536), (128, 1e4, 1 << 20), (64, 5e5, 1 << 22), (48, 1e4, 8192),
    (8, 1e4, 8192), (6, 1e4, 8192), (4, 1e4, 8192), (2, 1e4, 8192), (2, 1e4, 40), (128, 1e4, 8192),
    (128, 1e6, 32768), (64, 1e4, 100)])
@pytest.mark.parametrize("factor,fast,slow", [(16.0, 32.0, 1.0), (4.0, 40.0, 2.5), (1.0, 32.0, 1.0)])
def test_ends_of_the_ramp(rot, base, context, factor, fast, slow):
    freq, m = va.rope_ladder(rot, base, "parts", factor, context, fast, slow)
    full, _ = va.rope_ladder(rot, base)
    assert m == pytest.approx(1 + 0.1 * math.log(factor))
    # 1e-13: some ten roundings of 2^-53 and the ramp's ends, which are whole numbers
    for f, x, s in zip(full, freq, shares(rot, base, context, factor, fast, slow)):
        assert x == pytest.approx((1 - s) * f + s * f / factor, rel=1e-13, abs=0)
        if context * f / (2 * math.pi) > slow and factor > 1:
            assert x > f / factor * (1 + 1e-9)   # more turns than the slow end's: not divided in full


def test_lowest_frequency_of_a_long_context():
    """45 + 24 of a ramp of 25 pairs: the slow end, pair 69.1, is past the last of 64."""
    freq, _ = va.rope_ladder(128, 1e4, "parts", 16.0, 131072)
    full, _ = va.rope_ladder(128, 1e4)
    assert freq[-1] / full[-1] == pytest.approx(1 - 18 / 25 * 15 / 16, rel=1e-12, abs=0)


def test_short_ladders_of_their_own():
    plan = va.rope_plan(24, scaling="parts", factor=16.0, context=8192, sections=(2, 3, 7),
                        own_ladders=True)
    at = 0
    for n in (2, 3, 7):
        full, _ = va.rope_ladder(2 * n)
        for f, x, s in zip(full, plan.freq[at:at + n], shares(2 * n, 1e4, 8192, 16.0, 32.0, 1.0)):
            assert x == pytest.approx((1 - s) * f + s * f / 16, rel=1e-13, abs=0)
        at += n
    assert plan.freq[1] / va.rope_ladder(4)[0][1] == pytest.approx(1 - 0.5 * 15 / 16, rel=1e-12, abs=0)
