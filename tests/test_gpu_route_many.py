"""Routing of more rows than are given a wavefront each, and what must not hang on how many there are."""
import pytest
import torch

import routing_ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
FEW = 2048                                            # rows up to which a call lays them out for latency


@pytest.mark.parametrize("N", [6, FEW + 3])
@pytest.mark.parametrize("E,groups", [(8, 2), (30, 3), (64, 4), (64, 16), (160, 8), (256, 8), (256, 64), (1000, 5)])
def test_groups_with_infinite_biases(N, E, groups):
    """Two experts of bias +inf are worth as much as one: the lower group on a tie."""
    x = torch.randn(N, E, generator=torch.Generator().manual_seed(E))
    size, sample = E // groups, torch.arange(N) if N < 10 else torch.tensor([0, 1, 63, 1024, FEW - 1, FEW, FEW + 2])
    last = (groups - 1) * size
    for places in ([(1, INF), (last, INF), (last + 1, INF)], [(0, INF), (1, INF), (last, INF)], [(1, NAN), (last, INF), (last + 1, INF)], [(1, INF), (last, NAN), (last + 1, INF)]):
        b = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(1))
        for e, v in places:
            b[e] = v
        for score in ("softmax", "sigmoid"):
            how = dict(score=score, groups=groups, groups_kept=1, group_best=2)
            got = sp24.sp24_moe_route(x.cuda(), 2, bias=b.cuda(), **how)
            want = routing_ref.route(x[sample], 2, bias=b, **how)[0]
            assert torch.equal(got.ids.cpu()[sample].long(), want.long()), (places, score)
