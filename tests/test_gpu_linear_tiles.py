"""Every tile shape that layers and experts' rows run on, both layouts, with a partial last step of K and ragged rows and columns: sampled tokens
over all features against 64 bits, with the whole epilogue.  (Which shape takes which sizes is a matter of speed; the sizes here are the smallest found for each.)"""
import pytest
import torch

import layers_ref as ref
from paper_2104_08378_amd import sp24
from test_gpu_linear import check, expected, segments, strided, values, weights

pytestmark = pytest.mark.gpu

F16, BF16, F32, I8, F8 = torch.float16, torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn
WIDE, NARROW = (F16, BF16), (I8, F8)

# (types, M, N, K, layout)
LAYERS = [
    (WIDE, 63, 3, 96, "canonical"), (NARROW, 63, 20, 96, "canonical"), (WIDE, 63, 45, 96, "canonical"), (NARROW, 64, 3, 64, "tiled"),
    (WIDE, 64, 20, 64, "tiled"), (NARROW, 64, 45, 64, "tiled"),                                                # K split over a workgroup
    (WIDE, 8200, 3, 96, "canonical"), (NARROW, 8200, 3, 96, "canonical"), (WIDE, 512, 70, 64, "tiled"), (NARROW, 512, 70, 64, "tiled"),   # 64 x 32
    (WIDE, 3001, 300, 608, "canonical"), (NARROW, 1001, 1030, 1120, "canonical"), (WIDE, 3008, 300, 576, "tiled"), (NARROW, 3008, 300, 1088, "tiled"),   # 128 x 64
    (WIDE, 730, 2100, 96, "canonical"), (NARROW, 8200, 200, 96, "canonical"), (WIDE, 6016, 200, 64, "tiled"), (NARROW, 6016, 200, 64, "tiled"),   # 128 x 128
    (WIDE, 3001, 700, 2144, "canonical"), (NARROW, 3001, 700, 4192, "canonical"), (WIDE, 6016, 513, 2112, "tiled"), (NARROW, 6016, 513, 4160, "tiled"),   # six stages
    (WIDE, 8200, 4100, 96, "canonical"), (NARROW, 8200, 4100, 96, "canonical"), (WIDE, 8192, 700, 64, "tiled"), (NARROW, 8192, 700, 64, "tiled"),   # 256 x 128
    (WIDE, 2050, 4100, 608, "canonical"), (NARROW, 2050, 4100, 608, "canonical"), (WIDE, 8192, 1030, 576, "tiled"), (NARROW, 8192, 1030, 576, "tiled"),   # 256 x 256
]


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("case", range(len(LAYERS)))
def test_layers(case, which):
    types, M, N, K, layout = LAYERS[case]
    dtype, out = types[which], (BF16, F16)[which]
    g = torch.Generator().manual_seed(case)
    V, meta, W = weights(g, M, K, dtype, layout)
    x = values(g, (N, K), dtype).cuda()
    narrow = dtype in NARROW
    ws = (0.5 + torch.rand(M, generator=g)).cuda() / (1024 * K ** 0.5) if narrow else None
    xs = (0.5 + torch.rand(N, generator=g)).cuda() if narrow else None
    b = torch.randn(M, generator=g).cuda()
    at = torch.unique(torch.cat([torch.tensor([0, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, N - 2, N - 1]).clamp(0, N - 1), torch.randint(0, N, (30,), generator=g)])).cuda()
    z, err = expected(W, x[at], ws, None if xs is None else xs[at], b, "gelu", dtype, K)
    for pitch in (0, 3):                                          # rows of the result on 16-byte boundaries or not
        r, zt = strided(torch.randn(N, M, generator=g).to(out), pitch, 0)[0], strided(torch.zeros(N, M).to(out), pitch, 0)[0]
        y, buf = strided(torch.zeros(N, M).to(out), pitch, 0)
        sp24.sp24_linear(V, meta, x, out, w_scale=ws, x_scale=xs, bias=b, act="gelu", residual=r, preact=zt, layout=layout, out=y)
        check(y[at], zt[at], z, err, "gelu", r[at], str((LAYERS[case][1:], dtype)))
        if pitch:
            assert bool(torch.isnan(buf[:N * (M + pitch)].view(N, M + pitch)[:, M:]).all()), "written between the rows"
    # the same numbers whatever the result's rows are aligned to, in every row
    y0 = sp24.sp24_linear(V, meta, x, out, w_scale=ws, x_scale=xs, bias=b, act="gelu", residual=r.contiguous(), layout=layout)
    assert torch.equal(y0, y)


# (types, lengths in sixteens, M, K, layout)
EXPERTS = [
    (WIDE, [1, 2, 1], 63, 96, "canonical"), (NARROW, [1, 2, 1], 64, 64, "tiled"), (WIDE, [1, 2, 1], 2050, 96, "canonical"), (NARROW, [1, 2, 1], 2050, 96, "canonical"),
    (WIDE, [1, 2, 1], 2080, 64, "tiled"), (NARROW, [1, 2, 1], 2080, 64, "tiled"), (WIDE, [20, 33, 7], 1001, 608, "canonical"), (NARROW, [40, 1, 60, 13], 513, 2144, "canonical"),
    (WIDE, [40, 1, 60, 13], 512, 576, "tiled"), (NARROW, [40, 1, 60, 13], 512, 1088, "tiled"), (WIDE, [150] * 4, 161, 96, "canonical"), (NARROW, [70, 1, 130], 513, 96, "canonical"),
    (WIDE, [64] * 8, 160, 64, "tiled"), (NARROW, [150] * 4, 160, 64, "tiled"), (WIDE, [40, 1, 60, 13], 4100, 2144, "canonical"), (NARROW, [40, 1, 60, 13], 4100, 4192, "canonical"),
    (WIDE, [40, 1, 60, 13], 4096, 2112, "tiled"), (NARROW, [40, 1, 60, 13], 4096, 4160, "tiled"),
]


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("case", range(len(EXPERTS)))
def test_experts(case, which):
    types, lengths, M, K, layout = EXPERTS[case]
    dtype, out = types[which], (BF16, F16)[which]
    g = torch.Generator().manual_seed(case)
    offsets, o, R = segments(lengths, 1)
    E = len(lengths)
    V, meta, W = weights(g, E * M, K, dtype, layout)
    x = values(g, (R, K), dtype).cuda()
    narrow = dtype in NARROW
    ws = (0.5 + torch.rand(E * M, generator=g)).cuda() / (1024 * K ** 0.5) if narrow else None
    xs = (0.5 + torch.rand(R, generator=g)).cuda() if narrow else None
    b = torch.randn(E * M, generator=g).cuda()
    zt, y = (torch.full((R, M), float("nan"), dtype=out, device="cuda") for _ in range(2))
    sp24.sp24_linear_grouped(V, meta, x, offsets, out, w_scale=ws, x_scale=xs, bias=b, act="silu", preact=zt, layout=layout, out=y)
    for e in range(E):
        if o[e + 1] == o[e]:
            continue
        rows = slice(e * M, (e + 1) * M)
        at = torch.unique(torch.cat([torch.tensor([o[e], o[e + 1] - 1]), torch.randint(o[e], o[e + 1], (10,), generator=g)])).cuda()
        z, err = expected(W[rows], x[at], None if ws is None else ws[rows], None if xs is None else xs[at], b[rows], "silu", dtype, K)
        check(y[at], zt[at], z, err, "silu", None, str((EXPERTS[case][1:], dtype, e)))
    assert bool((y[o[-1]:] == 0).all()) and bool((zt[o[-1]:] == 0).all()) and bool(torch.isfinite(y[:o[-1]].float()).all())
