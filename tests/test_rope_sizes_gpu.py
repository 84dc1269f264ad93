"""Rotary positions of sizes that change how the work is dealt out: more tokens than one dimension
of a launch holds."""
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
