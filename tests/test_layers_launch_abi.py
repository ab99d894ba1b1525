"""Host-only: layers of more tiles than a launch has workgroups are refused before any launch (the addresses are made up)."""
import pytest

from paper_2104_08378_amd import sp24

SHAPE = 2
A, B, C, D, E = (i << 44 for i in range(1, 6))
M, N, K = 1 << 22, 1 << 17, 256                       # 2^39 results: 2^23 tiles of 256 x 256, 512 threads each


@pytest.mark.parametrize("i", [sp24.BF16, sp24.F16, sp24.I8, sp24.F8])
@pytest.mark.parametrize("m,n,k,layout,x", [
    (M, N, K, sp24.TILED, C), (M, N, K, sp24.CANONICAL, C), (1 << 30, 900, 64, sp24.CANONICAL, C), (M, N, 32, sp24.CANONICAL, C + 4),
    (1 << 20, 1 << 19, K, sp24.TILED, C + 4), (1, 1 << 30, 64, sp24.CANONICAL, C)])
def test_layers(m, n, k, layout, x, i):
    L = sp24.lib()
    assert L.sp24_linear(A, B, x, D, m, n, k, k, m, 0, 0, 0, 0, 0, 0, 0, 0, i, sp24.BF16, layout, None) == SHAPE


@pytest.mark.parametrize("layout", [sp24.TILED, sp24.CANONICAL])
def test_experts(layout):
    L = sp24.lib()
    for x in (C, C + 4):
        assert L.sp24_linear_grouped(A, B, x, D, E, 4, M, N, K, K, M, 0, 0, 0, 0, 0, 0, sp24.BF16, sp24.BF16, layout, None) == SHAPE
    for n, k in ((N, 128), (N - 8, 128), (1 << 18, 64)):
        assert L.sp24_gemm_dense_grouped(A, B, D, E, 4, M, n, k, k, n, n, sp24.BF16, sp24.BF16, None) == SHAPE
