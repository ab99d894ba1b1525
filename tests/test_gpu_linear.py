"""Layers on the sparse product -- alone, and for experts' rows -- and the gradients through their epilogues, against 64 bits.

Tolerances.  A sum of K / 2 kept products in binary32 is off by less than (K / 2 + 4) 2^-24 of the sum of their magnitudes (8-bit floats: the
matrix instruction drops low bits, 2^-13 of that sum; integers: exact up to 2^24 2^-24 of it); scales and bias add two roundings; the activations, whose slopes stay
below 1.13, a few units of 2^-24 of their argument."""
import pytest
import torch

import layers_ref as ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

F16, BF16, F32, I8, F8 = torch.float16, torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn
NAN = float("nan")


def values(g, shape, dtype, sigma=1.0):
    x = torch.randn(shape, generator=g) * sigma
    if dtype == I8:
        return (x * 32).round().clamp(-127, 127).to(I8)
    return x.to(dtype)


def strided(t, pitch, offset, fill=None):
    """The same matrix on the GPU in a buffer of NaN (ones, for integers) with this row pitch and first element."""
    N, K = t.shape
    raw = torch.full((offset + N * (K + pitch) + 16,), 1 if t.dtype == I8 else 0, dtype=t.dtype if t.dtype != F8 else torch.uint8, device="cuda")
    raw.fill_(0x7F if t.dtype == F8 else 1 if t.dtype == I8 else NAN)
    view = raw[offset:offset + N * (K + pitch)].view(N, K + pitch)[:, :K]
    view.copy_(t.view(torch.uint8) if t.dtype == F8 else t)
    return (raw.view(F8)[offset:offset + N * (K + pitch)].view(N, K + pitch)[:, :K] if t.dtype == F8 else view), raw


def weights(g, M, K, dtype, layout):
    W = values(g, (M, K), dtype, 1.0 if dtype in (I8, F8) else (2.0 / K) ** 0.5).cuda()
    V, meta = sp24.sp24_compress(W, layout=layout)
    return V, meta, ref.d(sp24.sp24_decompress(V, meta, layout=layout))


def expected(W, x, w_scale, x_scale, b, act, dtype, K):
    """(z, the error that z may have)."""
    x = ref.d(x)
    z, room = x @ W.t(), x.abs() @ W.abs().t()
    s = torch.ones(1, 1, dtype=torch.float64)
    if w_scale is not None:
        s = s * ref.d(w_scale)[None]
    if x_scale is not None:
        s = s * ref.d(x_scale)[:, None]
    unit = 2.0 ** -13 if dtype == F8 else 2.0 ** -24 if dtype == I8 else (K / 2 + 4) * 2.0 ** -24
    z, err = z * s, room * s * (unit + 3 * 2.0 ** -24)
    if b is not None:
        z, err = z + ref.d(b)[None], err + ref.d(b)[None].abs() * 2.0 ** -23
    return z, err + z.abs() * 2.0 ** -23


def check(y, zt, z, err, act, r, what):
    if zt is not None:
        ref.close(zt, z, err, what + " z")
    want = ref.act(z, act)
    err = 1.13 * err + z.abs() * 12 * 2.0 ** -24
    if r is not None:
        want, err = want + ref.d(r), err + (want.abs() + ref.d(r).abs()) * 2.0 ** -24
    ref.close(y, want, err, what)


# (M, N, K, layout, row pitch of X, its first element): each with the kernel that takes it
CASES = [
    (32, 1, 64, "tiled", 0, 0), (64, 16, 128, "tiled", 0, 0), (96, 33, 192, "canonical", 0, 0),          # few columns, K split
    (37, 5, 64, "canonical", 0, 0), (1, 1, 32, "canonical", 0, 0), (45, 64, 352, "canonical", 0, 0),     # rows that no tile divides
    (64, 7, 128, "tiled", 5, 3), (33, 70, 96, "canonical", 1, 1), (100, 40, 160, "canonical", 16, 1),    # rows of X at any address
    (256, 17, 2048, "tiled", 0, 0), (512, 100, 1024, "tiled", 16, 0), (8, 300, 64, "canonical", 0, 0),
    (100, 20, 48, "canonical", 0, 0), (700, 333, 1072, "canonical", 0, 0), (2100, 3000, 144, "canonical", 0, 0), (1030, 90, 400, "canonical", 3, 1),   # X through registers
    (5000, 1100, 176, "canonical", 0, 0), (60, 5000, 80, "canonical", 0, 0), (4128, 1040, 320, "tiled", 1, 1),
    (2560, 300, 256, "tiled", 0, 0), (3000, 130, 192, "canonical", 0, 0), (4096, 70, 128, "tiled", 0, 0),      # tiles of 64 to 128
    (4100, 1030, 128, "canonical", 0, 0), (4096, 2100, 320, "tiled", 0, 0), (8224, 1100, 64, "tiled", 0, 0), (11072, 20, 128, "tiled", 0, 0),
]


@pytest.mark.parametrize("dtype", [F16, BF16, I8, F8])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_linear(case, dtype):
    M, N, K, layout, pitch, offset = CASES[case]
    K = -(-K // 32) * 32 if dtype in (I8, F8) else K
    g = torch.Generator().manual_seed(case)
    V, meta, W = weights(g, M, K, dtype, layout)
    x, keep = strided(values(g, (N, K), dtype), pitch, offset)
    narrow = dtype in (I8, F8)
    outs = [BF16 if narrow else dtype, F32, F16 if dtype != F16 else BF16]
    for i, (act, with_bias, with_r, with_z, with_s) in enumerate([("none", False, False, False, False), ("gelu", True, True, True, True),
                                                                  ("silu", True, False, False, True), ("relu", False, True, True, False)]):
        out = outs[i % 3] if M * N < 1 << 20 else outs[0]
        # (results of unit size where a 16-bit float could not hold the integers)
        ws = (0.5 + torch.rand(M, generator=g)).cuda() / (1024 * K ** 0.5 if dtype == I8 else K ** 0.5) if narrow and (with_s or dtype == I8) else None
        xs = (0.5 + torch.rand(N, generator=g)).cuda() if narrow and with_s else None
        b = torch.randn(M, generator=g).cuda() if with_bias else None
        r = strided(torch.randn(N, M, generator=g).to(out), 3, 1)[0] if with_r else None
        zt = strided(torch.full((N, M), 7.0).to(out), 0, 2 if with_r else 0)[0] if with_z else None
        y, buf = strided(torch.full((N, M), 7.0).to(out), 5 if with_r else 0, 3 if with_r else 0)
        got = sp24.sp24_linear(V, meta, x, out, w_scale=ws, x_scale=xs, bias=b, act=act, residual=r, preact=zt, layout=layout, out=y)
        assert got.data_ptr() == y.data_ptr()
        z, err = expected(W, x, ws, xs, b, act, dtype, K)
        check(y, zt, z, err, act, r, (CASES[case], dtype, out, act).__str__())
        outside = torch.ones_like(buf, dtype=torch.bool)
        first = 3 if with_r else 0
        p = M + (5 if with_r else 0)
        outside[first:first + N * p].view(N, p)[:, :M] = False
        assert bool(torch.isnan(buf[outside]).all()), "written outside the result"
        again = sp24.sp24_linear(V, meta, x, out, w_scale=ws, x_scale=xs, bias=b, act=act, residual=r, layout=layout)
        assert torch.equal(again, y)


def test_a_large_layer_on_samples():
    """Tiles of 256 x 256 with several rounds of workgroups: sampled rows and features."""
    M, N, K = 4096, 8192, 512
    g = torch.Generator().manual_seed(1)
    for dtype, out in ((BF16, BF16), (I8, BF16), (F16, F32), (F8, F16)):
        V, meta, W = weights(g, M, K, dtype, "tiled")
        x = values(g, (N, K), dtype).cuda()
        ws = torch.full((M,), 1 / (1024 * K ** 0.5), device="cuda") if dtype == I8 else None
        b, r = torch.randn(M, generator=g).cuda(), torch.randn(N, M, generator=g).to(out).cuda()
        y = sp24.sp24_linear(V, meta, x, out, w_scale=ws, bias=b, act="gelu", residual=r, layout="tiled")
        at = torch.cat([torch.tensor([0, 1, 31, 32, 127, 128, 255, 256, 4095, 4096, N - 1]), torch.randint(0, N, (40,), generator=g)])
        z, err = expected(W, x[at.cuda()], ws, None, b, "gelu", dtype, K)
        check(y[at.cuda()], None, z, err, "gelu", r[at.cuda()], str(dtype))


def test_residual_in_place_and_on_another_stream():
    g = torch.Generator().manual_seed(2)
    V, meta, _ = weights(g, 512, 256, BF16, "tiled")
    x, r = values(g, (50, 256), BF16).cuda(), values(g, (50, 512), BF16).cuda()
    want = sp24.sp24_linear(V, meta, x, BF16, act="silu", residual=r, layout="tiled")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        mine = r.clone()
        got = sp24.sp24_linear(V, meta, x, BF16, act="silu", residual=mine, layout="tiled", out=mine)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want) and got.data_ptr() == mine.data_ptr()


def test_removed_positions_take_no_part_and_kept_ones_do():
    M, K, N = 64, 128, 20
    W = torch.zeros(M, K, dtype=BF16, device="cuda")
    W[:, 0::4], W[:, 1::4] = 1.0, 2.0
    for layout in ("canonical", "tiled"):
        V, meta = sp24.sp24_compress(W, layout=layout)
        x = torch.ones(N, K, dtype=BF16, device="cuda")
        x[3, 2], x[4, 3], x[5, 0], x[6, 1] = float("inf"), NAN, float("inf"), NAN
        y = sp24.sp24_linear(V, meta, x, BF16, bias=torch.ones(M, device="cuda"), act="relu", layout=layout)
        assert bool((y[:5] == 97).all()) and bool(torch.isinf(y[5]).all()) and bool(torch.isnan(y[6]).all()) and bool((y[7:] == 97).all())


def test_nothing_to_do():
    g = torch.Generator().manual_seed(2)
    V, meta, _ = weights(g, 64, 64, BF16, "tiled")
    assert tuple(sp24.sp24_linear(V, meta, torch.empty(0, 64, dtype=BF16, device="cuda"), BF16, layout="tiled").shape) == (0, 64)


def test_refusals():
    g = torch.Generator().manual_seed(2)
    V, meta, _ = weights(g, 64, 64, BF16, "tiled")
    x, ok = values(g, (8, 64), BF16).cuda(), dict(layout="tiled")
    one = torch.ones(64, device="cuda")
    for bad in (dict(act="tanh"), dict(bias=one[:63]), dict(bias=one.to(BF16)), dict(residual=torch.zeros(8, 63, dtype=BF16, device="cuda")),
                dict(residual=torch.zeros(8, 64, device="cuda")), dict(preact=torch.zeros(7, 64, dtype=BF16, device="cuda")),
                dict(out=torch.zeros(8, 64, device="cuda")), dict(residual=torch.zeros(8, 64, dtype=BF16))):
        with pytest.raises(ValueError):
            sp24.sp24_linear(V, meta, x, BF16, **ok, **bad)
    with pytest.raises(ValueError):
        sp24.sp24_linear(V, meta, x[:, :32], BF16, **ok)
    with pytest.raises(ValueError):
        sp24.sp24_linear(V, meta, x.to(F16), BF16, **ok)
    for bad, status in ((dict(w_scale=one), 4), (dict(x_scale=torch.ones(8, device="cuda")), 4)):       # scales are the 8-bit types'
        with pytest.raises(sp24.Sp24Error) as e:
            sp24.sp24_linear(V, meta, x, BF16, **ok, **bad)
        assert e.value.status == status
    with pytest.raises(sp24.Sp24Error) as e:
        sp24.sp24_linear(V, meta, x, torch.int32, **ok)
    assert e.value.status == 4
    y = torch.zeros(9, 64, dtype=BF16, device="cuda")
    with pytest.raises(sp24.Sp24Error) as e:                              # the residual one row off: not in place
        sp24.sp24_linear(V, meta, x, BF16, residual=y[1:], out=y[:8], **ok)
    assert e.value.status == 2
    with pytest.raises(sp24.Sp24Error) as e:
        sp24.sp24_linear(V, meta, x, BF16, preact=y[:8], out=y[:8], **ok)
    assert e.value.status == 2


# ---- gradients through the epilogue ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("N,M,pitch,offset", [(1, 1, 0, 0), (16, 64, 0, 0), (70, 33, 3, 1), (129, 200, 8, 0), (64, 513, 0, 5), (1000, 72, 0, 0), (2050, 2049, 0, 0), (1030, 4104, 8, 0)])
def test_gradient_through_the_epilogue(N, M, pitch, offset, act, dtype):
    g = torch.Generator().manual_seed(N + M)
    dy, z = strided(values(g, (N, M), dtype), pitch, offset)[0], strided(values(g, (N, M), dtype, 2.0), pitch, offset)[0]
    dz, dzt, db = sp24.sp24_linear_backward(dy, None if act == "none" else z, act)
    want = ref.d(dy) * ref.slope(ref.d(z), act)
    err = ref.d(dy).abs() * (12 * 2.0 ** -24) * (1 + ref.d(z).abs())
    if act == "none":
        assert dz is dy
    else:
        ref.close(dz, want, err, "dz")
    assert torch.equal(dzt, dz.t())
    ref.close(db, want.sum(0), err.sum(0) + want.abs().sum(0) * (N + 4) * 2.0 ** -24, "db")


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_slopes_against_differences(act):
    """Far out as well, where a factor of the formula overflows."""
    z = torch.cat([torch.linspace(-12, 12, 401), torch.tensor([-60000.0, -31.0, 31.0, 60000.0])]).to(F16)[None].cuda()
    dz, _, _ = sp24.sp24_linear_backward(torch.ones_like(z), z, act)
    x, e = ref.d(z), 1e-6
    far = lambda t: ref.act(t.clamp(-40, 40), act) + (t - t.clamp(-40, 40)).clamp(min=0)  # noqa: E731
    want = (far(x + e) - far(x - e)) / (2 * e)
    if act == "relu":
        want = torch.where(x.abs() <= e, (x > 0).double(), want)      # (a difference across the corner is no slope)
    ref.close(dz, want, 2e-6, act)
    wide = torch.tensor([[3e38, -3e38, NAN]], dtype=BF16, device="cuda")
    slope = sp24.sp24_linear_backward(torch.ones_like(wide), wide, act)[0][0]
    assert float(slope[0]) == 1 and float(slope[1]) == 0 and bool(torch.isnan(slope[2]))


def test_no_rows_have_no_gradient():
    none = torch.empty(0, 64, dtype=BF16, device="cuda")
    dz, dzt, db = sp24.sp24_linear_backward(none, none, "gelu")
    assert tuple(dz.shape) == (0, 64) and tuple(dzt.shape) == (64, 0) and bool((db == 0).all())


# ---- experts' rows ---------------------------------------------------------------------------------------------

def segments(lengths, extra=0):
    """offsets of segments of these lengths (in sixteens), and the number of rows."""
    o = torch.tensor([0] + list(lengths)).cumsum(0) * 16
    return o.to(torch.int32).cuda(), o.tolist(), int(o[-1]) + 16 * extra


GROUPS = [
    # lengths in sixteens, rows behind the last, M, K, layout
    ([1], 0, 32, 64, "tiled"), ([1, 0, 2, 1], 1, 64, 128, "tiled"), ([0, 0, 0], 2, 64, 64, "tiled"), ([3, 5, 0, 9], 0, 100, 96, "canonical"),
    ([1] * 70, 3, 32, 64, "tiled"), ([0] * 40 + [4] + [0] * 90 + [1, 7], 0, 96, 192, "canonical"), ([20, 33, 7], 2, 512, 256, "tiled"),
    ([70, 1, 130], 1, 1024, 128, "tiled"), ([3, 0, 40, 9], 2, 70, 80, "canonical"), ([20, 50, 1, 100], 1, 1030, 144, "canonical"), ([1, 2], 1, 33, 16, "canonical"), ([2, 1, 0, 3, 1, 1, 2, 1], 4, 2048, 512, "tiled"), ([40] * 8, 0, 256, 64, "canonical"), ([64, 60], 0, 4096, 128, "tiled"),
]


@pytest.mark.parametrize("dtype", [F16, BF16, I8, F8])
@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_experts_rows(case, dtype):
    lengths, extra, M, K, layout = GROUPS[case]
    K = -(-K // 32) * 32 if dtype in (I8, F8) else K
    g = torch.Generator().manual_seed(case)
    offsets, o, R = segments(lengths, extra)
    E = len(lengths)
    V, meta, W = weights(g, E * M, K, dtype, layout)
    x = values(g, (R, K), dtype).cuda()
    narrow = dtype in (I8, F8)
    for act, with_bias, with_z, out in (("none", False, False, BF16 if narrow else dtype), ("silu", True, True, F32)):
        ws = (0.5 + torch.rand(E * M, generator=g)).cuda() / (1024 * K ** 0.5) if narrow else None
        xs = (0.5 + torch.rand(R, generator=g)).cuda() if narrow else None
        b = torch.randn(E * M, generator=g).cuda() if with_bias else None
        zt, y = (torch.full((R, M), NAN, dtype=out, device="cuda") for _ in range(2))
        sp24.sp24_linear_grouped(V, meta, x, offsets, out, w_scale=ws, x_scale=xs, bias=b, act=act, preact=zt if with_z else None, layout=layout, out=y)
        for e in range(E):
            part, rows = slice(o[e], o[e + 1]), slice(e * M, (e + 1) * M)
            z, err = expected(W[rows], x[part], None if ws is None else ws[rows], None if xs is None else xs[part], None if b is None else b[rows], act, dtype, K)
            check(y[part], zt[part] if with_z else None, z, err, act, None, str((GROUPS[case][2:], dtype, e)))
        assert bool((y[o[-1]:] == 0).all()) and (not with_z or bool((zt[o[-1]:] == 0).all()))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lengths,M,N,out32", [([1, 0, 2], 33, 8, False), ([3, 5, 9], 130, 200, True), ([0, 0], 64, 64, False), ([8, 1, 0, 33], 256, 136, False),
                                               ([70], 300, 520, True)])
def test_weights_gradient_of_experts(lengths, M, N, out32, dtype):
    g = torch.Generator().manual_seed(M)
    offsets, o, R = segments(lengths, 1)
    A, B = values(g, (M, R), dtype).cuda(), values(g, (R, N), dtype).cuda()
    D = sp24.sp24_gemm_dense_grouped(A, B, offsets, F32 if out32 else dtype)
    for e in range(len(lengths)):
        a, b = ref.d(A)[:, o[e]:o[e + 1]], ref.d(B)[o[e]:o[e + 1]]
        ref.close(D[e], a @ b, (a.abs() @ b.abs()) * (16 * lengths[e] + 4) * 2.0 ** -24, str(e))


@pytest.mark.parametrize("lengths", [[1, 0, 5, 2], [0, 0], [9]])
def test_bias_gradient_of_experts(lengths):
    g = torch.Generator().manual_seed(1)
    offsets, o, R = segments(lengths, 1)
    M = 72
    dy, z = values(g, (R, M), BF16).cuda(), values(g, (R, M), BF16).cuda()
    dz, dzt, db = sp24.sp24_linear_backward(dy, z, "silu", offsets=offsets)
    want = ref.d(dy) * ref.slope(ref.d(z), "silu")
    assert tuple(db.shape) == (len(lengths), M) and torch.equal(dzt, dz.t())
    for e in range(len(lengths)):
        part = want[o[e]:o[e + 1]]
        ref.close(db[e], part.sum(0), part.abs().sum(0) * (16 * lengths[e] + 30) * 2.0 ** -24 + len(part) * 2.0 ** -22, str(e))


def test_layer_gradient_against_differences():
    """<c, Y> of a layer in 64 bits by central differences along a direction of X, bias and the kept weights, against the gradients that the
    calls give: through the epilogue, the compressed transpose, and the masked dense product."""
    g = torch.Generator().manual_seed(4)
    M, K, N, dtype = 64, 128, 32, F16
    P = sp24.sp24_prune_transposable(values(g, (M, K), dtype, 0.2).cuda())
    V, meta = sp24.sp24_compress(P, layout="tiled")
    back = sp24.sp24_compress(P.t().contiguous(), layout="tiled")
    x, b, c = values(g, (N, K), dtype).cuda(), torch.randn(M, generator=g).cuda(), values(g, (N, M), dtype).cuda()
    z = torch.empty(N, M, dtype=dtype, device="cuda")
    sp24.sp24_linear(V, meta, x, dtype, bias=b, act="gelu", preact=z, layout="tiled")
    dz, dzt, db = sp24.sp24_linear_backward(c, z, "gelu")
    dx = sp24.sp24_linear(*back, dz, F32, layout="tiled")
    dW = sp24.sp24_mask_apply(sp24.sp24_gemm_dense(dzt, x, dtype, b_order="n"), meta, layout="tiled")
    W, X, B, C = ref.d(P), ref.d(x), ref.d(b), ref.d(c)
    for seed in range(3):
        gg = torch.Generator().manual_seed(seed)
        vx, vb, vw = (torch.randn(s, generator=gg).double() for s in ((N, K), (M,), (M, K)))
        vw, e = vw * (W != 0), 1e-5
        value = lambda t: (ref.act((X + t * vx) @ (W + t * vw).t() + B + t * vb, "gelu") * C).sum()  # noqa: E731
        got = (ref.d(dx) * vx).sum() + (ref.d(db) * vb).sum() + (ref.d(dW) * vw).sum()
        slope = (value(e) - value(-e)) / (2 * e)
        # z, dz and dW are rounded to 11 bits: independent errors of 2^-12 at most, over the square root of the sum of squares
        spread = ((ref.d(dx) * vx).square().sum() + (ref.d(db) * vb).square().sum() + (ref.d(dW) * vw).square().sum()).sqrt()
        assert abs(float(got - slope)) <= 6 * 2.0 ** -10 * float(spread)
