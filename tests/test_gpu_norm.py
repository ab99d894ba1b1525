"""The norm of rows, its 8-bit rows, the quantisation alone and the gradients, against 64 bits.

Tolerances.  rstd: the mean of squares is a sum of H terms in binary32, H / 64 of them in a row at most, so it is off by less than
(H / 64 + 16) 2^-24, half of that after the root; y adds four roundings.  Gradients: sums of products of H (N) terms likewise, relative to
the sum of their magnitudes."""
import pytest
import torch

import layers_ref as ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

F16, BF16, F32, I8, F8 = torch.float16, torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn
EPS = 1e-6


def rows(g, N, H, dtype, pitch=0, offset=0, sigma=1.0):
    """[N, H] of normal values inside a buffer of NaN: a row pitch and a first element that nothing is aligned to."""
    buf = torch.full((offset + N * (H + pitch) + 8,), float("nan"), dtype=dtype, device="cuda")
    t = buf[offset:offset + N * (H + pitch)].view(N, H + pitch)[:, :H]
    t.copy_((torch.randn(N, H, generator=g) * sigma).to(dtype))
    return t


def rel(H):
    return (H / 64 + 16) * 2.0 ** -25 + 4 * 2.0 ** -24


@pytest.mark.parametrize("out", [F16, BF16, F32])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,H,pitch,offset,residual", [
    (1, 1, 0, 0, False), (3, 7, 0, 0, True), (5, 64, 8, 0, True), (2, 333, 0, 3, True), (17, 512, 3, 1, False), (4, 2048, 0, 0, True),
    (1100, 520, 0, 0, True), (1030, 2056, 8, 0, True), (2, 8200, 0, 0, True), (3, 16384, 0, 8, False), (1, 32768, 0, 0, True), (0, 64, 0, 0, True)])
def test_norm(N, H, pitch, offset, residual, dtype, out):
    g = torch.Generator().manual_seed(N * 1000 + H)
    x, w = rows(g, N, H, dtype, pitch, offset), (1 + 0.2 * torch.randn(H, generator=g)).cuda()
    r = rows(g, N, H, dtype, 2 * pitch, offset) if residual else None
    y = rows(g, N, H, out, pitch, offset)
    whole = y.untyped_storage()
    n = sp24.sp24_rmsnorm(x, w, EPS, residual=r, out_dtype=out, want_rstd=True, out=y)
    h, rstd, want = ref.norm(x, w, EPS, r)
    ref.close(n.rstd, rstd, rel(H) * rstd, "rstd")
    ref.close(y, want, rel(H) * want.abs() + 2.0 ** -24 * ref.d(w).abs() * rstd[:, None], "y")
    if residual:
        ref.close(n.hidden, h, h.abs() * 2.0 ** -24, "h")
    else:
        assert n.hidden is None
    assert n.scale is None
    flat = torch.empty(0, dtype=out, device="cuda").set_(whole)
    inside = torch.zeros(flat.numel(), dtype=torch.bool, device="cuda")
    inside[offset:offset + N * (H + pitch)].view(N, H + pitch)[:, :H] = True
    assert bool(torch.isnan(flat[~inside]).all()), "written outside the rows"


@pytest.mark.parametrize("out", [I8, F8])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,H,pitch,offset,alone", [
    (1, 1, 0, 0, False), (5, 7, 0, 3, True), (3, 100, 4, 0, False), (9, 512, 0, 0, True), (2, 1000, 0, 1, False), (1040, 520, 0, 0, False),
    (1040, 520, 8, 0, True), (3, 4096, 0, 0, False), (2, 8200, 0, 0, True), (2, 32768, 0, 0, False), (2, 65536, 0, 0, True), (1030, 64, 0, 0, True)])
def test_rows_of_8_bits(N, H, pitch, offset, alone, dtype, out):
    g = torch.Generator().manual_seed(N * 1000 + H)
    x, w = rows(g, N, H, dtype, pitch, offset), (1 + 0.2 * torch.randn(H, generator=g)).cuda()
    if alone:
        want, err = ref.d(x), 2.0 ** -22
        q, scale = sp24.sp24_quantize_rows(x, out)
    else:
        r = rows(g, N, H, dtype, pitch, offset)
        n = sp24.sp24_rmsnorm(x, w, EPS, residual=r, out_dtype=out)
        q, scale, want, err = n.y, n.scale, ref.norm(x, w, EPS, r)[2], rel(H) + 2.0 ** -21
    assert q.dtype == out and scale.dtype == F32 and tuple(scale.shape) == (N,)
    top = want.abs().amax(1).clamp(min=2.0 ** -100)
    ref.close(scale, top / ref.TOP[out], err * top / ref.TOP[out], "scale")
    s, q = ref.d(scale)[:, None], ref.d(q)
    assert bool((q.abs().amax(1) == ref.TOP[out]).all()), "the largest code is the type's"
    # half a code; half a unit of three fraction bits, or half the smallest step
    step = 0.5 * s if out == I8 else torch.maximum(want.abs() * 2.0 ** -4, s * 2.0 ** -10)
    assert bool(((q * s - want).abs() <= step * (1 + 1e-5) + 2 * err * top[:, None]).all())


def test_rows_that_are_zero_tiny_or_not_numbers():
    x = torch.zeros(6, 100, device="cuda")
    x[1] = 1e-38
    x[2, 3] = float("nan")
    x[3, 5] = float("inf")
    x[4, 99] = -5.0
    x[5] = 1e-3
    for out in (I8, F8):
        q, scale = sp24.sp24_quantize_rows(x, out)
        q = ref.d(q)
        assert bool((q[:2] == 0).all()) and bool(torch.isfinite(scale[:2]).all()) and bool((scale[:2] > 0).all())
        assert torch.isnan(scale[2]) and torch.isinf(scale[3])
        assert float(q[4, 99]) == -ref.TOP[out] and int((q[4] != 0).sum()) == 1
        assert bool((q[5] == ref.TOP[out]).all())
    w = torch.ones(100, device="cuda")
    n = sp24.sp24_rmsnorm(x, w, EPS, out_dtype=I8, want_rstd=True)
    assert torch.isnan(n.scale[2]) and torch.isnan(n.scale[3]) and float(n.rstd[0]) == pytest.approx(1e3, rel=1e-6)
    y = sp24.sp24_rmsnorm(x, w, EPS, out_dtype=BF16).y
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isfinite(y[4:]).all())


@pytest.mark.parametrize("size,eps", [(2.0 ** -120, 1e-36), (2.0 ** -110, 1e-30), (2.0 ** -90, 1e30), (2.0 ** -60, 1e-6), (2.0 ** 60, 1e-6)])
def test_small_and_large_rows_of_8_bits(size, eps):
    """Rows far from 1 and what eps makes of them; their squares may be nothing in binary32, as eps alone then says."""
    x = (torch.tensor([[1.0, -0.5, 0.25, 0.0, 0.75, -1.0, 0.125, 0.5]]) * size).cuda()
    w = torch.ones(8, device="cuda")
    y = sp24.sp24_rmsnorm(x, w, eps, out_dtype=F32).y
    for out in (I8, F8):
        n = sp24.sp24_rmsnorm(x, w, eps, out_dtype=out)
        want = ref.d(y)
        top = max(float(want.abs().max()), 2.0 ** -100)
        assert float(n.scale[0]) == pytest.approx(top / ref.TOP[out], rel=1e-6)
        exact = want / (top / ref.TOP[out])
        room = 0.5 if out == I8 else torch.maximum(exact.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10))
        assert bool(((ref.d(n.y) - exact).abs() <= room + 1e-4).all()), (size, eps, n.y)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_norm_in_place_on_the_residual(dtype):
    g = torch.Generator().manual_seed(5)
    x, r, w = rows(g, 37, 1000, dtype), rows(g, 37, 1000, dtype), torch.randn(1000, generator=g).cuda()
    want = sp24.sp24_rmsnorm(x, w, EPS, residual=r)
    stream = r.clone()
    n = sp24.sp24_rmsnorm(x, w, EPS, residual=stream, hidden=stream)
    assert torch.equal(n.y, want.y) and torch.equal(stream, want.hidden) and n.hidden.data_ptr() == stream.data_ptr()
    own = x.clone()
    n = sp24.sp24_rmsnorm(own, w, EPS, residual=r, out=own)
    assert torch.equal(own, want.y)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,H,pitch,offset,extra", [
    (1, 1, 0, 0, False), (3, 7, 0, 3, True), (65, 100, 4, 0, True), (4, 513, 0, 1, False), (700, 1024, 0, 0, True), (1500, 72, 8, 0, True),
    (9, 8192, 0, 0, False), (3, 8200, 0, 0, True), (2, 32768, 0, 0, True)])
def test_norm_gradients(N, H, pitch, offset, extra, dtype):
    g = torch.Generator().manual_seed(N + H)
    h, w = rows(g, N, H, dtype, pitch, offset), (1 + 0.2 * torch.randn(H, generator=g)).cuda()
    dy, dh = rows(g, N, H, dtype, 0, offset), rows(g, N, H, dtype, pitch, 0) if extra else None
    rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
    dx, dw = sp24.sp24_rmsnorm_backward(dy, h, w, rstd, dhidden=dh)
    want_dx, want_dw = ref.norm_grad(dy, h, w, rstd, dh)
    v, gw, hh = ref.d(rstd)[:, None], (ref.d(dy) * ref.d(w)).abs(), ref.d(h).abs()
    sums = (H / 64 + 20) * 2.0 ** -24
    ref.close(dx, want_dx, v * (gw * 2.0 ** -22 + hh * v * v * (gw * hh).mean(1, keepdim=True) * (sums + 2.0 ** -22)) + want_dx.abs() * 2.0 ** -23, "dx")
    ref.close(dw, want_dw, (ref.d(dy).abs() * hh * v).sum(0) * (N + 4) * 2.0 ** -24, "dw")
    again = sp24.sp24_rmsnorm_backward(dy, h, w, rstd, dhidden=dh)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_norm_gradients_against_differences():
    """The directional derivative of <c, y> in 64 bits, by central differences, against the kernel's gradients in binary32."""
    g = torch.Generator().manual_seed(3)
    N, H = 6, 300
    x, w, c = torch.randn(N, H, generator=g), 1 + 0.2 * torch.randn(H, generator=g), torch.randn(N, H, generator=g)
    n = sp24.sp24_rmsnorm(x.cuda(), w.cuda(), EPS, want_rstd=True)
    dx, dw = sp24.sp24_rmsnorm_backward(c.cuda(), x.cuda(), w.cuda(), n.rstd)
    for seed in range(4):
        gg = torch.Generator().manual_seed(100 + seed)
        vx, vw, e = torch.randn(N, H, generator=gg).double(), torch.randn(H, generator=gg).double(), 1e-5
        value = lambda t: (ref.norm(x.double() + t * vx, w.double() + t * vw, EPS)[2] * c.double()).sum()  # noqa: E731
        slope = (value(e) - value(-e)) / (2 * e)
        got = (ref.d(dx) * vx).sum() + (ref.d(dw) * vw).sum()
        assert abs(float(got - slope)) <= 1e-4 * float((ref.d(dx) * vx).abs().sum()) / H ** 0.5


@pytest.mark.parametrize("N,H,out", [(9000, 4096, F8), (8300, 1032, BF16), (33000, 72, I8), (9001, 1024, F16)])
def test_more_rows_than_workgroups(N, H, out):
    """Workgroups that take several rows: the last ones and some others."""
    g = torch.Generator().manual_seed(N)
    x, w = torch.randn(N, H, generator=g).to(BF16).cuda(), (1 + 0.2 * torch.randn(H, generator=g)).cuda()
    n = sp24.sp24_rmsnorm(x, w, EPS, residual=x, out_dtype=out, want_rstd=True)
    at = torch.cat([torch.arange(N - 40, N), torch.arange(0, N, 997), torch.arange(8180, 8200)]).cuda()
    h, rstd, want = ref.norm(x[at], w, EPS, x[at])
    ref.close(n.rstd[at], rstd, rel(H) * rstd, "rstd")
    ref.close(n.hidden[at], h, h.abs() * 2.0 ** -24, "h")
    if out in (I8, F8):
        s, q, top = ref.d(n.scale[at])[:, None], ref.d(n.y[at]), want.abs().amax(1)[:, None]
        ref.close(n.scale[at], top[:, 0] / ref.TOP[out], (rel(H) + 2.0 ** -21) * top[:, 0] / ref.TOP[out], "scale")
        step = 0.5 * s if out == I8 else torch.maximum(want.abs() * 2.0 ** -4, s * 2.0 ** -10)
        assert bool(((q * s - want).abs() <= step * (1 + 1e-5) + 2 * (rel(H) + 2.0 ** -21) * top).all())
    else:
        ref.close(n.y[at], want, rel(H) * want.abs() + 2.0 ** -24 * ref.d(w).abs() * rstd[:, None], "y")
    # and the gradients, whose workgroups take several rows each
    dx, dw = sp24.sp24_rmsnorm_backward(x, n.hidden, w, n.rstd)
    want_dx, _ = ref.norm_grad(x[at], n.hidden[at], w, n.rstd[at])
    ref.close(dx[at], want_dx, 2.0 ** -17 * want_dx.abs().amax(1, keepdim=True), "dx")
    dy, hh, v = (t.double() for t in (x, n.hidden, n.rstd[:, None]))
    ref.close(dw, (dy * hh * v).sum(0).cpu(), ((dy * hh * v).abs().sum(0) * (N + 4) * 2.0 ** -24).cpu(), "dw")


def test_no_rows():
    w = torch.ones(64, device="cuda")
    none = torch.empty(0, 64, dtype=BF16, device="cuda")
    n = sp24.sp24_rmsnorm(none, w, EPS, out_dtype=I8)
    assert tuple(n.y.shape) == (0, 64) and n.scale.numel() == 0
    dx, dw = sp24.sp24_rmsnorm_backward(none, none, w, torch.empty(0, device="cuda"))
    assert tuple(dx.shape) == (0, 64) and bool((dw == 0).all())


def test_refusals():
    x, w = torch.randn(4, 64, device="cuda", dtype=BF16), torch.ones(64, device="cuda")
    with pytest.raises(ValueError):
        sp24.sp24_rmsnorm(x, w[:63])
    with pytest.raises(ValueError):
        sp24.sp24_rmsnorm(x, w.to(BF16))
    with pytest.raises(ValueError):
        sp24.sp24_rmsnorm(x, w, residual=x[:3])
    with pytest.raises(ValueError):
        sp24.sp24_rmsnorm(x, w, residual=x.float())
    with pytest.raises(ValueError):
        sp24.sp24_rmsnorm(x.t(), torch.ones(4, device="cuda"))
    with pytest.raises(ValueError):
        sp24.sp24_rmsnorm(x.cpu(), w)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(sp24.Sp24Error) as e:
            sp24.sp24_rmsnorm(x, w, eps)
        assert e.value.status == 2
    with pytest.raises(sp24.Sp24Error):
        sp24.sp24_rmsnorm(x, w, out_dtype=torch.int32)
    buffer = torch.zeros(5, 64, device="cuda", dtype=BF16)
    with pytest.raises(sp24.Sp24Error):                           # a residual stream that overlaps the rows, not in place
        sp24.sp24_rmsnorm(buffer[:4], w, residual=buffer[1:], hidden=buffer[1:], out=buffer[:4])
    with pytest.raises(sp24.Sp24Error):
        sp24.sp24_quantize_rows(x, BF16)
    with pytest.raises(sp24.Sp24Error) as e:
        sp24.sp24_rmsnorm(torch.zeros(1, 32776, device="cuda"), torch.ones(32776, device="cuda"))
    assert e.value.status == 2
    with pytest.raises(sp24.Sp24Error) as e:
        sp24.sp24_rmsnorm_backward(x, x, w, torch.ones(4, device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 2
