"""The in-place forms of the gradients, results and workspaces that the caller brings: bit for bit what the calls return without them."""
import pytest
import torch

from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

F16, BF16, F32, I8, F8 = torch.float16, torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn
NAN = float("nan")


def normal(g, *shape, dtype=BF16):
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def same(a, b):
    assert a.dtype == b.dtype and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def scratch(need):
    """Exactly what is asked for, at the end of a buffer, behind and in front of it a pattern that has to stay."""
    raw = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    return raw[32:32 + need], raw


def untouched(raw):
    assert bool((raw[:32] == 0xA5).all()) and bool((raw[-32:] == 0xA5).all())


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,H", [(3, 7), (70, 512), (900, 1024), (1100, 2048), (65, 333), (33, 8192), (5, 8200), (3, 20000)])
def test_norm_gradient_in_place(N, H, dtype):
    """Rows of whole chunks, a wavefront's and a workgroup's, and ragged ones."""
    g = torch.Generator().manual_seed(N + H)
    given = dict(dY=normal(g, N, H, dtype=dtype), hidden=normal(g, N, H, dtype=dtype), dhidden=normal(g, N, H, dtype=dtype))
    w, rstd = normal(g, H, dtype=F32), torch.rand(N, generator=g).cuda() + 0.5
    call = lambda t, **more: sp24.sp24_rmsnorm_backward(t["dY"], t["hidden"], w, rstd, dhidden=t["dhidden"], **more)  # noqa: E731
    dx, dw = call(given)
    for name in given:
        mine = {k: v.clone() for k, v in given.items()}
        got = call(mine, out=mine[name])
        assert got[0].data_ptr() == mine[name].data_ptr()
        same(got[0], dx), same(got[1], dw)
        for other in given:
            if other != name:
                same(mine[other], given[other])
    ws, raw = scratch(sp24.lib().sp24_rmsnorm_backward_workspace_bytes(N, H))
    pitched = torch.full((N, H + 8), NAN, dtype=dtype, device="cuda")
    got = call(given, workspace=ws, out=pitched[:, :H])
    same(got[0], dx), same(got[1], dw), untouched(raw)
    assert bool(torch.isnan(pitched[:, H:]).all())


def layer_gradient(dY, Z, dZ, dZt, db, ws, need, act, dtype):
    N, M = dY.shape
    p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    status = sp24.lib().sp24_linear_backward(dY.data_ptr(), p(Z), p(dZ), p(dZt), p(db), M, N, M, M, M, N, act, None, 0, {F16: sp24.F16, BF16: sp24.BF16}[dtype],
                                             p(ws), need, torch.cuda.current_stream().cuda_stream)
    assert status == 0


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,M,act", [(70, 33, "gelu"), (129, 200, "relu"), (1030, 4104, "silu"), (64, 513, "none"), (1000, 72, "none")])
def test_gradient_of_a_layers_result_in_place(N, M, act, dtype):
    """dZ on dY and on Z (tiles of 64 and of 128 values), with the transpose and the bias's gradient and without."""
    g = torch.Generator().manual_seed(N + M)
    dy, z = normal(g, N, M, dtype=dtype), None if act == "none" else normal(g, N, M, dtype=dtype)
    dz, dzt, db = sp24.sp24_linear_backward(dy, z, act)
    need, code = sp24.lib().sp24_linear_backward_workspace_bytes(M, N, 0), {"none": 0, "relu": 1, "gelu": 2, "silu": 3}[act]
    for on in ("dY", "Z") if z is not None else ("dY",):
        for more in (True, False):
            mine = dict(dY=dy.clone(), Z=None if z is None else z.clone())
            ws, raw = scratch(need)
            t, b = (torch.full((M, N), NAN, dtype=dtype, device="cuda"), torch.full((M,), NAN, device="cuda")) if more else (None, None)
            layer_gradient(mine["dY"], mine["Z"], mine[on], t, b, ws if more else None, need if more else 0, code, dtype)
            same(mine[on], dz), untouched(raw)
            if more:
                same(t, dzt), same(b, db)
            if on == "Z":
                same(mine["dY"], dy)
            elif z is not None:
                same(mine["Z"], z)
    ws, raw = scratch(need)
    for a, b in zip(sp24.sp24_linear_backward(dy, z, act, workspace=ws), (dz, dzt, db)):
        same(a, b)
    untouched(raw)


def routed(g, N, topk, E):
    ids = torch.randint(-1, E, (N, topk), generator=g, dtype=torch.int32).cuda()
    return ids, sp24.sp24_moe_sort(ids, E)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,topk,E,H", [(1, 1, 4, 5), (40, 2, 8, 512), (300, 3, 5, 1001), (17, 4, 64, 2056)])
def test_gradients_of_the_combination_in_place(N, topk, E, H, dtype):
    g = torch.Generator().manual_seed(N + H)
    _, (offsets, slots, rows) = routed(g, N, topk, E)
    R = rows.numel()
    dout, y, weights = normal(g, N, H, dtype=dtype), normal(g, R, H, dtype=dtype), torch.rand(N, topk, generator=g).cuda()
    dy, dw = sp24.sp24_moe_combine_backward(dout, y, slots, rows, weights)
    mine = y.clone()
    got = sp24.sp24_moe_combine_backward(dout, mine, slots, rows, weights, out=mine)
    assert got[0].data_ptr() == mine.data_ptr()
    same(mine, dy), same(got[1], dw)
    pitched = torch.full((R, H + 3), NAN, dtype=dtype, device="cuda")
    got = sp24.sp24_moe_combine_backward(dout, y, slots, rows, weights, out=pitched[:, :H])
    same(got[0], dy), same(got[1], dw)
    assert bool(torch.isnan(pitched[:, H:]).all())
    stream = dout.clone()                                           # the residual's own buffer
    same(sp24.sp24_moe_combine(y, slots, weights, residual=stream, out=stream), sp24.sp24_moe_combine(y, slots, weights, residual=dout))


def test_results_and_workspaces_of_the_caller():
    g = torch.Generator().manual_seed(0)
    ids = torch.randint(0, 8, ((1 << 17) + 100, 1), generator=g, dtype=torch.int32).cuda()
    ws, raw = scratch(sp24.lib().sp24_moe_sort_workspace_bytes(ids.numel(), 8))
    for a, b in zip(sp24.sp24_moe_sort(ids, 8, workspace=ws), sp24.sp24_moe_sort(ids, 8)):
        same(a, b)
    untouched(raw)
    offsets = torch.tensor([0, 16, 16, 96], dtype=torch.int32, device="cuda")
    A, B = normal(g, 100, 112), normal(g, 112, 72)
    D = torch.full((3, 100, 72), NAN, device="cuda")
    got = sp24.sp24_gemm_dense_grouped(A, B, offsets, F32, out=D)
    assert got.data_ptr() == D.data_ptr()
    same(D, sp24.sp24_gemm_dense_grouped(A, B, offsets, F32))
    x = normal(g, 50, 333)
    for out in (I8, F8):
        q = torch.empty(50, 340, dtype=torch.uint8, device="cuda").fill_(0x55)
        got, scale = sp24.sp24_quantize_rows(x, out, out=q.view(out)[:, :333])
        want = sp24.sp24_quantize_rows(x, out)
        same(got, want[0]), same(scale, want[1])
        assert bool((q[:, 333:] == 0x55).all())
    dy, z = normal(g, 96, 72), normal(g, 96, 72)
    ws, raw = scratch(sp24.lib().sp24_linear_backward_workspace_bytes(72, 96, 1))
    for a, b in zip(sp24.sp24_linear_backward(dy, z, "gelu", offsets=offsets, workspace=ws), sp24.sp24_linear_backward(dy, z, "gelu", offsets=offsets)):
        same(a, b)
    untouched(raw)
