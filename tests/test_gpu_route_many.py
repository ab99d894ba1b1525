"""Routing of more rows than are given a wavefront each, and what must not hang on how many there are."""
import math

import numpy as np
import pytest
import torch

import routing_ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
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


@pytest.mark.parametrize("E", [20, 32, 64, 100, 128, 256])
def test_a_row_has_the_same_experts_among_few_and_among_many(E):
    """Every row has the same logits, each in an order of its own, and the biases of experts a and b make of their scores the same to within a bit of binary64 (that of a
    all but 2^-24 of the difference, that of b the rest): which of the two is chosen tells one order of the softmax's sum from another."""
    N, a, b = 3 * FEW, 3, E - 2
    g = torch.Generator().manual_seed(E)
    rest = torch.tensor([e for e in range(E) if e not in (a, b)])
    x = torch.zeros(N, E)
    x[:, rest] = (0.5 * torch.randn(E - 2, generator=g) - 4)[torch.rand(N, E - 2, generator=g).argsort(1)]
    x[:, a] = 1
    others = float(x[0, rest].double().exp().sum())

    def biases(l):
        total = others + math.e + math.exp(l)
        p, q = math.e / total, math.exp(l) / total
        of_a = float(np.float32(q - p))
        of_b = float(np.float32(math.fsum([p, of_a, -q])))
        return abs(math.fsum([p, of_a, -q, -of_b])), l, of_a, of_b
    _, x[:, b], of_a, of_b = min(biases(k / 512) for k in range(400))
    bias = torch.zeros(E)
    bias[a], bias[b] = of_a, of_b
    x, bias = x.cuda(), bias.cuda()
    for how in (dict(topk=1), dict(topk=min(E, 64), want_scores=True)):
        many = sp24.sp24_moe_route(x, bias=bias, **how)
        for first in range(0, N, FEW):
            few = sp24.sp24_moe_route(x[first:first + FEW], bias=bias, **how)
            for p, q in zip(many[:3], few[:3]):
                assert p is None or torch.equal(p[first:first + FEW], q)
