"""The gradient of a layer's weights from any number of tokens: the dense product of dZ transposed and X, whose inner dimension that number
is, against 64 bits.

Tolerance: a sum of K products in binary32 is off by less than (K + 4) 2^-24 of the sum of their magnitudes; the result is rounded once."""
import pytest
import torch

import layers_ref as ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
NAN = float("nan")


def strided(t, pitch, offset):
    """The same matrix on the GPU inside a buffer of NaN, rows `pitch` apart, from element `offset` on."""
    N, K = t.shape
    raw = torch.full((offset + (N + 2) * pitch + 16,), NAN, dtype=t.dtype, device="cuda")
    view = raw[offset:offset + N * pitch].view(N, pitch)[:, :K]
    view.copy_(t)
    return view


def product(M, N, K, dtype, out, b_pitch=None, b_offset=0, spare=0):
    g = torch.Generator().manual_seed(M + N + K)
    a, b = torch.randn(M, K, generator=g).to(dtype), torch.randn(K, N, generator=g).to(dtype)
    A, B = strided(a, -(-K // 8) * 8 + spare, 0), strided(b, b_pitch or N, b_offset)
    D = sp24.sp24_gemm_dense(A, B, out, b_order="n")
    ref.close(D, ref.d(a) @ ref.d(b), (ref.d(a).abs() @ ref.d(b).abs()) * (K + 4) * 2.0 ** -24, str((M, N, K, dtype, out)))
    assert torch.equal(sp24.sp24_gemm_dense(A, B, out, b_order="n"), D)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("K", [1, 2, 7, 8, 9, 15, 17, 24, 63, 65, 77, 127, 200, 509, 1021])
def test_any_number_of_tokens(K, dtype):
    product(70, 40, K, dtype, F32)
    product(200, 264, K, dtype, dtype, spare=16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,N", [(1540, 1288), (1920, 1664), (2304, 2048), (4096, 1920), (4096, 2304), (66600, 104)])
def test_every_tile(M, N, dtype):
    product(M, N, 77, dtype, dtype)
    product(M, N, 197, dtype, F32)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,N,pitch,offset", [(70, 45, 45, 0), (33, 64, 67, 1), (1, 1, 1, 0), (300, 1411, 1411, 0), (2100, 201, 203, 3), (5, 8, 9, 1)])
def test_rows_of_x_at_any_address(M, N, pitch, offset, dtype):
    for K in (1, 3, 15, 17, 31, 75, 130, 509):
        product(M, N, K, dtype, F32 if K % 2 else dtype, pitch, offset)


def test_no_tokens():
    A, B = torch.empty(33, 0, dtype=BF16, device="cuda"), torch.empty(0, 72, dtype=BF16, device="cuda")
    D = sp24.sp24_gemm_dense(A, B, F32, b_order="n", out=torch.full((33, 72), NAN, device="cuda"))
    assert bool((D == 0).all())
    B = torch.empty(0, 5, dtype=BF16, device="cuda")
    assert bool((sp24.sp24_gemm_dense(A, B, BF16, b_order="n", out=torch.full((33, 5), NAN, dtype=BF16, device="cuda")) == 0).all())


class Declines:
    """Stands in for the native module and declines every call."""

    def __getattr__(self, name):
        return lambda *a: None


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("N", [0, 1, 5, 8, 33, 509, 1000])
def test_from_the_gradient_of_a_layers_result(N, act, native, monkeypatch):
    """The transpose that sp24_linear_backward gives goes into the product as it is, then the pattern."""
    if not native:
        monkeypatch.setattr(sp24, "_host", Declines())
    g = torch.Generator().manual_seed(N)
    M, K = 96, 128
    W = sp24.sp24_prune((torch.randn(M, K, generator=g) * 0.1).to(BF16).cuda())
    meta = sp24.sp24_compress(W, layout="tiled")[1]
    dy, z, x = (torch.randn(N, n, generator=g).to(BF16).cuda() for n in (M, M, K))
    dz, dzt, db = sp24.sp24_linear_backward(dy, z, act)
    assert tuple(dzt.shape) == (M, N) and torch.equal(dzt, dz.t()) and dzt.data_ptr() % 16 == 0 and (N == 0 or dzt.stride(0) % 8 == 0)
    dW = sp24.sp24_mask_apply(sp24.sp24_gemm_dense(dzt, x, BF16, b_order="n"), meta, layout="tiled")
    want, room = ref.d(dz).t() @ ref.d(x), ref.d(dz).abs().t() @ ref.d(x).abs()
    kept = ref.d(W) != 0
    ref.close(dW, want * kept, room * kept * (N + 4) * 2.0 ** -24, "dW")


def test_weight_gradient_against_differences():
    """<c, Y> of a layer on 37 tokens in 64 bits, by central differences along a direction of the kept weights."""
    g = torch.Generator().manual_seed(4)
    M, K, N = 64, 128, 37
    P = sp24.sp24_prune((torch.randn(M, K, generator=g) * 0.2).to(F16).cuda())
    V, meta = sp24.sp24_compress(P, layout="tiled")
    x, b, c = torch.randn(N, K, generator=g).to(F16).cuda(), torch.randn(M, generator=g).cuda(), torch.randn(N, M, generator=g).to(F16).cuda()
    z = torch.empty(N, M, dtype=F16, device="cuda")
    sp24.sp24_linear(V, meta, x, F16, bias=b, act="silu", preact=z, layout="tiled")
    dzt = sp24.sp24_linear_backward(c, z, "silu")[1]
    dW = sp24.sp24_mask_apply(sp24.sp24_gemm_dense(dzt, x, F16, b_order="n"), meta, layout="tiled")
    W, X, B, C = ref.d(P), ref.d(x), ref.d(b), ref.d(c)
    for seed in range(3):
        vw, e = torch.randn(M, K, generator=torch.Generator().manual_seed(seed)).double() * (W != 0), 1e-5
        value = lambda t: (ref.act(X @ (W + t * vw).t() + B, "silu") * C).sum()  # noqa: E731
        slope = (value(e) - value(-e)) / (2 * e)
        # z, dz and dW are rounded to 11 bits: independent errors of 2^-12 at most, over the square root of the sum of squares
        assert abs(float((ref.d(dW) * vw).sum() - slope)) <= 6 * 2.0 ** -10 * float((ref.d(dW) * vw).square().sum().sqrt())


def test_other_products_keep_the_rule():
    x = lambda *s, dtype=BF16: torch.zeros(*s, device="cuda").to(dtype)  # noqa: E731
    for call in (lambda: sp24.sp24_gemm_dense(x(16, 24), x(16, 24), F32), lambda: sp24.sp24_gemm_dense(x(16, 16, dtype=torch.int8), x(16, 16, dtype=torch.int8), torch.int32, b_order="n"),
                 lambda: sp24.sp24_gemm_dense_splitk(x(16, 24), x(24, 16), F32, b_order="n"), lambda: sp24.sp24_gemm_dense(x(16, 0), x(16, 0), F32)):
        with pytest.raises(sp24.Sp24Error) as e:
            call()
        assert e.value.status == 2
    with pytest.raises(sp24.Sp24Error) as e:                               # rows of A off 16 bytes
        sp24.sp24_gemm_dense(x(16, 25), x(25, 16), F32, b_order="n")
    assert e.value.status == 3
