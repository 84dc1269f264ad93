"""Refusals of vecattn_cache_gather and vecattn_cache_gather_wide: no call below reaches the GPU."""
import ctypes

import pytest

from paper_2603_29494_amd import _lib

INVALID = 1
FAKE = 0x100000   # 16-byte aligned address that validation rejects before any use


@pytest.mark.parametrize("bad", [
    dict(M_out=7), dict(M_out=(1 << 30) + 1), dict(M_out=0), dict(M_out=-1), dict(flags=2),
    dict(mass=None), dict(mass_out=None), dict(M=0), dict(idx=None), dict(kept=None),
    dict(budget=0, M_out=8), dict(cols=0), dict(to_cols=0), dict(B=0)])
def test_gather_wide_rejects_bad_arguments(bad):
    c = _lib.CacheDesc(FAKE, 8, 2, 128, 64, 4)
    a = dict(cols=4, B=2, idx=FAKE, kept=FAKE, budget=8, to_cols=4, mass=FAKE, M=256, mass_out=FAKE,
             M_out=8, flags=0)
    a.update(bad)
    assert _lib.load().vecattn_cache_gather_wide(
        ctypes.byref(c), FAKE, a["cols"], a["B"], a["idx"], a["kept"], a["budget"], ctypes.byref(c),
        FAKE, a["to_cols"], a["mass"], a["M"], a["mass_out"], a["M_out"], a["flags"],
        None) == INVALID


@pytest.mark.parametrize("budget", [(1 << 29) + 1, 1 << 30])
def test_gather_refuses_more_slots_than_a_launch_holds(budget):
    c, f = _lib.CacheDesc(FAKE, 8, 2, 128, 64, 4), ctypes.byref
    lib, unsupported = _lib.load(), 2
    assert lib.vecattn_cache_gather(f(c), FAKE, 4, 2, FAKE, FAKE, budget, f(c), FAKE, 4, None, 0,
                                    None, 0, None) == unsupported
    assert lib.vecattn_cache_gather_wide(f(c), FAKE, 4, 2, FAKE, FAKE, budget, f(c), FAKE, 4, FAKE,
                                         256, FAKE, 1 << 30, 0, None) == unsupported
