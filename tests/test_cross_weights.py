"""The bounds of cross_weights tell weights of one bf16 from weights of two."""
import pytest

import cross_weights as cw


@pytest.mark.parametrize("D,Nq,Nk", [(64, 1, 5), (128, 4, 33), (64, 8, 300)])
def test_bounds_see_the_second_part(D, Nq, Nk):
    q, k, v = cw.inputs(Nk, 2, 4, 2, Nq, Nk, D)
    o, _, bound, _ = cw.cross64(q, k, v)
    assert ((cw.rounded(q, k, v, 2).double() - o).abs() <= bound).all()
    over = (cw.rounded(q, k, v, 1).double() - o).abs() > bound
    assert over.sum() > 20
