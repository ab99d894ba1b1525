"""Routing of more rows than are given a wavefront each, and what must not hang on how many there are."""
import math

import numpy as np
import pytest
import torch

import layers_ref as ref
import routing_ref
from paper_2104_08378_amd import sp24
from test_gpu_route import expected

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


def rows(N, E, dtype, seed):
    """Logits of N rows: normal ones, and in places rows that are masked, infinite, NaN or full of ties."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, E, generator=g) * 2
    kind = torch.arange(N) % 11
    masked = torch.rand(N, E, generator=g) < 0.9
    x = torch.where((kind == 3)[:, None] & masked, -INF, x)
    x = torch.where((kind == 5)[:, None], x.round(), x)
    x[kind == 7] = torch.randint(18, 50, (int((kind == 7).sum()), E), generator=g).float()
    x[60::97, E // 2] = NAN
    x[61::97, E // 3] = INF
    x[62::97] = -INF
    x[63::97, 1:] = -INF
    return x.to(dtype)


# (groups of whole power-of-two runs of lanes and groups of any other size, of 2, 4 or 8 experts a lane)
MANY = [(8, (2, 4)), (16, (4, 16)), (20, (4, 10)), (32, (4, 32)), (64, (4, 64)), (100, (25, 5)), (128, (4, 128)), (160, (5, 8)), (256, (8, 256)), (512, (8, 512)), (1000, (125, 8))]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("E,groups", MANY)
def test_many_rows(E, groups, dtype):
    """All rows against calls of few of them, to the bit, and some against 64 bits."""
    N = FEW + 37
    x = rows(N, E, dtype, E)
    sample = torch.cat((torch.arange(0, 120), torch.arange(FEW - 3, N)))
    b = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(1))
    b[E // 4], b[E // 2 + 1] = -INF, b[0]
    dev, tiny = x.cuda(), (E + 16) * 2.0 ** -53
    topk = min(8, E // 2)
    hows = [dict(score="softmax", bias=b), dict(score="sigmoid", renormalise=False, scale=2.5)]
    for n in groups:
        kept = max(n // 2, -(-topk // (E // n)))
        hows += [dict(score="sigmoid", bias=b, groups=n, groups_kept=kept, group_best=2), dict(score="softmax", groups=n, groups_kept=kept, group_best=1)]
    for how in hows:
        on = dict(how, bias=how["bias"].cuda()) if "bias" in how else how
        got = sp24.sp24_moe_route(dev, topk, want_scores=True, want_load=True, **on)
        few = [sp24.sp24_moe_route(dev[i:i + FEW // 2], topk, want_scores=True, **on) for i in range(0, N, FEW // 2)]
        for a, part in zip(got[:3], zip(*few)):
            assert torch.equal(a.view(torch.int32), torch.cat(part[:len(few)]).view(torch.int32)), how
        ids, weights, scores, _ = routing_ref.route(x[sample], topk, **how)
        assert torch.equal(got.ids.cpu()[sample].long(), ids.long()), how
        ref.close(got.scores.cpu()[sample], scores, torch.nan_to_num(scores) * tiny, "scores")
        ref.close(got.weights.cpu()[sample], weights, torch.nan_to_num(weights.abs()) * tiny * 2, "weights")
        flat = got.ids.reshape(-1).long()
        assert torch.equal(got.load.long(), torch.bincount(flat[flat >= 0], minlength=E)), how


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("E,topk", [(8, 3), (16, 16), (20, 4), (32, 8), (64, 40), (100, 8), (128, 64), (160, 6), (256, 8), (1000, 10)])
def test_gradient_of_many_rows(E, topk, dtype, score):
    N = FEW + 5
    g = torch.Generator().manual_seed(E)
    x = (torch.randn(N, E, generator=g) * 2).to(dtype)
    x[::7, 0] = -INF
    ids = x.float().topk(topk, dim=1).indices.to(torch.int32)
    ids[1::5, 0], ids[2::50], ids[3::50, -1] = -1, -1, E
    dw, ds = torch.randn(N, topk, generator=g).cuda(), torch.randn(N, E, generator=g).cuda()
    for renormalise, d, scale in ((True, ds, 0.5), (True, None, 1.0), (False, ds, 2.5)):
        want, size = expected(x, ids, dw, d, score, renormalise, scale)
        got = sp24.sp24_moe_route_backward(x.cuda(), ids.cuda(), dw, score=score, renormalise=renormalise, scale=scale, dscores=d)
        # (as for few rows: a few thousand operations of 2^-53, and the rounding on the way to 32 bits)
        ref.close(got, want, size * 4096 * 2.0 ** -53 + want.abs() * 2.0 ** -24, str((E, topk, dtype, score, renormalise)))
