"""Window attention's gradients where many keys are sinks, by the parts that their tiles
are cut into: many, few and one. Against the float64 oracle with the window tests'
tolerances, and against cross attention where every key is a sink."""
import pytest
import torch

import paper_2609_23169_amd as ut
from test_gpu_swattn import check_case, draw, random_mask, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [(20, 0), (20, 7)])
@pytest.mark.parametrize("B,n,Hq,Hk,D,sinks", [(1, 1500, 2, 1, 64, 1500), (1, 1500, 2, 2, 128, 1499), (2, 900, 4, 2, 72, 700),
                                               (1, 2100, 1, 1, 128, 129), (1, 300, 2, 2, 64, 1 << 30)])
def test_many_sinks_match_oracle(B, n, Hq, Hk, D, sinks, window):
    check_case(50, B, n, n, Hq, Hk, D, window, sinks)
    check_case(51, B, n, n, Hq, Hk, D, window, sinks, random_mask(52, B, n))


def test_sinks_that_fill_the_chip_are_whole():
    """7,536 tiles of sinks, one part each: what cross attention gives."""
    q, k, v, do = draw(53, 2, 20000, 20000, 24, 24, 128)
    assert ut.ut_swattn_bwd_workspace_size(2, 20000, 20000, 24, 24, 128, (16, 3), 20000) == \
        ut.ut_swattn_bwd_workspace_size(2, 20000, 20000, 24, 24, 128, (16, 3), 0)
    o, lse, grads = run(q, k, v, do, 0.09, (16, 3), 20000)
    o2, lse2 = ut.xattn_fwd(q, k, v, 0.09)
    grads2 = ut.xattn_bwd(q, k, v, o2, do, lse2, 0.09)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for x, y in zip(grads, grads2):   # the same sums in the same order, but for the steps' first token
        assert (x.float() - y.float()).norm() <= 2.0 ** -8 * y.float().norm()
