"""Plans of rotary positions copied, saved and sent: plain values that come back the same."""
import copy
import ctypes
import io
import pickle

import pytest
import torch

import paper_2603_29494_amd as va


class Layer(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.plan = va.rope_plan(24, layout="interleaved", scaling="parts", factor=4.0,
                                 context=4096, sections=(3, 4, 5))
        self.w = torch.nn.Parameter(torch.zeros(3))


def saved(x):
    f = io.BytesIO()
    torch.save(x, f)
    f.seek(0)
    return torch.load(f, weights_only=False)   # what this test has just written


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x)),
                                   saved], ids=["copy", "deepcopy", "pickle", "save"])
def test_a_plan_comes_back_the_same(again):
    for plan in (va.rope_plan(64), Layer().plan):
        other = again(plan)
        assert other == plan and hash(other) == hash(plan) and repr(other) == repr(plan)
        assert other.axes == plan.axes
        for a, b in zip(other._specs, plan._specs):   # what calls are given, of memory of its own
            a, b = a._obj, b._obj
            assert (a.rot, a.layout, a.axes, a.flags, a.factor) == (b.rot, b.layout, b.axes, b.flags,
                                                                     b.factor)
            n = a.rot // 2
            assert a.freq[:n] == b.freq[:n] == list(plan.freq)
            assert a.axis[:n] == b.axis[:n] == list(plan.axis)
            assert ctypes.addressof(a.freq.contents) != ctypes.addressof(b.freq.contents)


def test_a_model_that_holds_a_plan():
    for other in (copy.deepcopy(Layer()), saved(Layer())):
        assert other.plan == Layer().plan
