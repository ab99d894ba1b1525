"""Tokens sorted by expert, gathered, combined, and the gradients of that, against a plain statement in 64 bits; whole numbers exactly."""
import pytest
import torch

import layers_ref as ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

F16, BF16, F32, I8, F8 = torch.float16, torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn


def choices(g, N, topk, E, dropped):
    ids = torch.randint(0, E, (N, topk), generator=g, dtype=torch.int32)
    if dropped:
        ids[torch.rand(N, topk, generator=g) < dropped] = -1
        ids[torch.rand(N, topk, generator=g) < dropped / 4] = E
        ids[torch.rand(N, topk, generator=g) < dropped / 8] = -2 ** 31
    return ids.cuda()


@pytest.mark.parametrize("N,topk,E,dropped", [
    (0, 2, 4, 0), (1, 1, 1, 0), (1, 2, 8, 0), (16, 2, 8, 0), (63, 1, 3, 0), (64, 1, 64, 0.3), (65, 1, 65, 0), (100, 4, 1024, 0.1), (700, 3, 7, 0.2),
    (1024, 1, 1, 0), (4096, 2, 8, 0), (4096, 4, 64, 0.05), (5461, 3, 128, 0), (16384, 1, 5, 0), (16385, 1, 1000, 0.1), (20000, 4, 33, 0), (30, 2, 4, 1.0),
    (65536, 2, 8, 0.1), (65536, 2, 9, 0), (131073, 1, 3, 0), (70001, 2, 700, 0.05),
])
def test_sort(N, topk, E, dropped):
    g = torch.Generator().manual_seed(N + E)
    ids = choices(g, N, topk, E, dropped)
    offsets, slots, rows = sp24.sp24_moe_sort(ids, E)
    o, s, r = ref.sort(ids.cpu(), E)
    assert rows.numel() == sp24.sp24_moe_rows(N * topk, E) == len(r)
    assert offsets.cpu().tolist() == o and slots.cpu().reshape(-1).tolist() == s and rows.cpu().tolist() == r


def test_sort_of_one_expert_only():
    """All choices on one expert, at either end; long runs of one key cross every wavefront and part."""
    for E, which in ((8, 0), (8, 7), (1024, 1023)):
        for N in (20000, 80000):
            ids = torch.full((N, 2), which, dtype=torch.int32, device="cuda")
            offsets, slots, rows = sp24.sp24_moe_sort(ids, E)
            assert torch.equal(slots.reshape(-1), torch.arange(2 * N, dtype=torch.int32, device="cuda")) and torch.equal(rows[:2 * N], slots.reshape(-1))
            assert bool((rows[2 * N:] == -1).all()) and offsets.cpu().tolist() == [0] * (which + 1) + [2 * N] * (E - which)


SHAPES = [(1, 1, 1, 8, 0, 0), (5, 2, 4, 7, 0, 0), (16, 2, 8, 64, 0.3, 0), (33, 3, 5, 1000, 0.2, 3), (300, 2, 8, 72, 0, 8), (64, 8, 16, 2056, 0.1, 0), (9, 1, 64, 4097, 0, 1),
          (700, 4, 32, 256, 0.05, 0)]


def padded(t, pitch):
    """The same rows with a pitch, NaN between them."""
    if t.element_size() == 1:
        buf = torch.full((t.shape[0], t.shape[1] + pitch), 0x7F, dtype=torch.uint8, device="cuda")
        buf[:, :t.shape[1]] = t.view(torch.uint8)
        return buf.view(t.dtype)[:, :t.shape[1]]
    buf = torch.full((t.shape[0], t.shape[1] + pitch), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


@pytest.mark.parametrize("dtype", [F16, BF16, F32, I8, F8])
@pytest.mark.parametrize("N,topk,E,H,dropped,pitch", SHAPES)
def test_gather(N, topk, E, H, dropped, pitch, dtype):
    g = torch.Generator().manual_seed(N + H)
    _, _, rows = sp24.sp24_moe_sort(choices(g, N, topk, E, dropped), E)
    x = torch.randn(N, H, generator=g)
    x = padded(((x * 32).clamp(-127, 127).to(I8) if dtype == I8 else x.to(dtype)).cuda(), pitch)
    xs, scales = sp24.sp24_moe_gather(x, rows, topk, scale=torch.arange(1.0, N + 1, device="cuda"))
    token = (rows.long() // topk).clamp(min=0)
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
    want = torch.where(rows[:, None] >= 0, x.contiguous().view(raw)[token], 0)
    assert torch.equal(xs.view(raw), want) and torch.equal(scales, torch.where(rows >= 0, token + 1.0, 0.0))
    assert torch.equal(sp24.sp24_moe_gather(x, rows, topk).view(raw), want)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("weighted,residual", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("N,topk,E,H,dropped,pitch", SHAPES)
def test_combine(N, topk, E, H, dropped, pitch, weighted, residual, dtype):
    g = torch.Generator().manual_seed(N + H)
    _, slots, rows = sp24.sp24_moe_sort(choices(g, N, topk, E, dropped), E)
    y = torch.randn(rows.numel(), H, generator=g).to(dtype).cuda()
    y[rows < 0] = float("nan")                                   # rows of no choice are not looked at
    y = padded(y, pitch)
    w = torch.rand(N, topk, generator=g).cuda() if weighted else None
    r = padded(torch.randn(N, H, generator=g).to(dtype).cuda(), 2 * pitch) if residual else None
    out = sp24.sp24_moe_combine(y, slots, weights=w, residual=r)
    part = torch.where(slots.cpu()[..., None] >= 0, ref.d(y)[slots.cpu().long().clamp(min=0)], 0.0) * (1 if w is None else ref.d(w)[..., None])
    want, size = part.sum(1), part.abs().sum(1)
    if residual:
        want, size = want + ref.d(r), size + ref.d(r).abs()
    ref.close(out, want, size * (topk + 1) * 2.0 ** -24, "out")
    if residual:
        mine = r.clone()
        assert sp24.sp24_moe_combine(y, slots, weights=w, residual=mine, out=mine).data_ptr() == mine.data_ptr() and torch.equal(mine, out)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,topk,E,H,dropped,pitch", SHAPES)
def test_combine_gradients(N, topk, E, H, dropped, pitch, dtype):
    g = torch.Generator().manual_seed(N + H)
    _, slots, rows = sp24.sp24_moe_sort(choices(g, N, topk, E, dropped), E)
    y = torch.randn(rows.numel(), H, generator=g).to(dtype).cuda()
    y[rows < 0] = float("nan")
    y, dout, w = padded(y, pitch), padded(torch.randn(N, H, generator=g).to(dtype).cuda(), pitch), torch.rand(N, topk, generator=g).cuda()
    dy, dw = sp24.sp24_moe_combine_backward(dout, y, slots, rows, w)
    token, choice = (rows.cpu().long() // topk).clamp(min=0), rows.cpu().long().clamp(min=0)
    live = (rows.cpu() >= 0)[:, None]
    want = torch.where(live, ref.d(dout)[token] * ref.d(w).reshape(-1)[choice][:, None], 0.0)
    ref.close(dy, want, 0.0, "dy")                                # one product, rounded to binary32 and to the type
    prod = torch.where(slots.cpu()[..., None] >= 0, ref.d(y)[slots.cpu().long().clamp(min=0)] * ref.d(dout)[:, None, :], 0.0)
    ref.close(dw, prod.sum(2), prod.abs().sum(2) * (H / 64 + 16) * 2.0 ** -24, "dweights")


def test_combine_gradients_against_differences():
    """The combination is linear in the rows and in the weights: a difference is the derivative."""
    g = torch.Generator().manual_seed(9)
    N, topk, E, H = 20, 3, 6, 40
    _, slots, rows = sp24.sp24_moe_sort(choices(g, N, topk, E, 0.1), E)
    y, w, c = (torch.randn(s, generator=g).cuda() for s in ((rows.numel(), H), (N, topk), (N, H)))
    vy, vw = torch.randn(y.shape, generator=g).cuda(), torch.randn(w.shape, generator=g).cuda()
    dy, dw = sp24.sp24_moe_combine_backward(c, y, slots, rows, w)
    part = lambda yy, ww: (torch.where(slots.cpu()[..., None] >= 0, yy[slots.cpu().long().clamp(min=0)] * ww[..., None], 0.0).sum(1) * ref.d(c)).sum()  # noqa: E731
    Y, W, VY, VW, e = ref.d(y), ref.d(w), ref.d(vy), ref.d(vw), 1e-3
    slope = (part(Y + e * VY, W + e * VW) - part(Y - e * VY, W - e * VW)) / (2 * e)
    got = (ref.d(dy) * VY).sum() + (ref.d(dw) * VW).sum()
    assert abs(float(got - slope)) <= 1e-5 * float((ref.d(dy) * VY).abs().sum() + (ref.d(dw) * VW).abs().sum())
    # and of the gathering, whose gradient is the combination without weights
    x = torch.randn(N, H, generator=g)
    xs = sp24.sp24_moe_gather(x.cuda(), rows, topk)
    assert float((ref.d(xs) * VY).sum()) == pytest.approx(float((ref.d(sp24.sp24_moe_combine(vy, slots)) * x.double()).sum()), rel=1e-5)


def test_nothing_has_a_row():
    slots, none = torch.full((5, 2), -1, dtype=torch.int32, device="cuda"), torch.empty(0, 64, dtype=BF16, device="cuda")
    x, w = torch.ones(5, 64, dtype=BF16, device="cuda"), torch.ones(5, 2, device="cuda")
    rows = torch.empty(0, dtype=torch.int32, device="cuda")
    assert bool((sp24.sp24_moe_combine(none, slots, w) == 0).all()) and torch.equal(sp24.sp24_moe_combine(none, slots, w, residual=x), x)
    dy, dw = sp24.sp24_moe_combine_backward(x, none, slots, rows, w)
    assert tuple(dy.shape) == (0, 64) and bool((dw == 0).all())
    xs, scales = sp24.sp24_moe_gather(torch.empty(0, 64, dtype=I8, device="cuda"), torch.full((16,), -1, dtype=torch.int32, device="cuda"), 2, scale=torch.empty(0, device="cuda"))
    assert bool((xs == 0).all()) and bool((scales == 0).all())


def test_refusals():
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    offsets, slots, rows = sp24.sp24_moe_sort(ids, 4)
    x, w = torch.zeros(4, 64, dtype=BF16, device="cuda"), torch.ones(4, 2, device="cuda")
    for bad in (lambda: sp24.sp24_moe_sort(ids.long(), 4), lambda: sp24.sp24_moe_sort(ids.cpu(), 4), lambda: sp24.sp24_moe_sort(ids.t(), 4),
                lambda: sp24.sp24_moe_gather(x, rows.long(), 2), lambda: sp24.sp24_moe_gather(x, rows, 2, scale=torch.ones(3, device="cuda")),
                lambda: sp24.sp24_moe_combine(x, slots.reshape(-1)), lambda: sp24.sp24_moe_combine(x, slots, weights=w[:3]),
                lambda: sp24.sp24_moe_combine(x, slots, residual=x.float()), lambda: sp24.sp24_moe_combine_backward(x.float(), x, slots, rows, w),
                lambda: sp24.sp24_moe_combine_backward(x, x, slots, rows, w)):
        with pytest.raises(ValueError):
            bad()
    for experts in (0, -3, 1025):
        with pytest.raises(sp24.Sp24Error) as e:
            sp24.sp24_moe_sort(ids, experts)
        assert e.value.status == 2
    with pytest.raises(sp24.Sp24Error) as e:
        sp24.sp24_moe_gather(x, rows, 0)
    assert e.value.status == 2
    with pytest.raises(sp24.Sp24Error) as e:
        sp24.sp24_moe_sort(torch.zeros((1 << 17) + 1, 1, dtype=torch.int32, device="cuda"), 64, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 2
