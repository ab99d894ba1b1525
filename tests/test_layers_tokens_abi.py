"""Host-only: which inner dimensions the dense product takes (no rows: nothing is launched; the addresses are made up)."""
from paper_2104_08378_amd import sp24

OK, SHAPE, ALIGN = 0, 2, 3
A, B, D = 0x10000000, 0x20000000, 0x30000000


def dense(M=0, N=64, K=509, lda=512, ldb=64, ldd=64, i=sp24.BF16, o=sp24.F32, bo=sp24.B_NMAJOR, a=A):
    return sp24.lib().sp24_gemm_dense(a, B, D, M, N, K, lda, ldb, ldd, i, o, bo, None)


def test_any_number_of_tokens():
    assert [dense(K=k) for k in (0, 1, 15, 16, 24, 509)] == [OK] * 6 and dense(i=sp24.F16) == OK
    assert dense(K=-1) == SHAPE and dense(M=64, K=509, lda=504) == SHAPE and dense(M=64, lda=509) == ALIGN and dense(M=64, a=A + 2) == ALIGN
    assert dense(bo=sp24.B_KMAJOR) == SHAPE and dense(i=sp24.F8) == SHAPE and dense(i=sp24.I8, o=sp24.I32) == SHAPE and dense(bo=sp24.B_KMAJOR, K=0) == SHAPE
    L = sp24.lib()
    assert L.sp24_gemm_dense_splitk(A, B, D, 0, 64, 509, 512, 64, 64, sp24.BF16, sp24.F32, sp24.B_NMAJOR, 0, 0, None) == SHAPE
    assert L.sp24_spmm(A, A, B, D, 0, 64, 509, 64, 64, sp24.BF16, sp24.F32, sp24.B_NMAJOR, sp24.CANONICAL, None) == SHAPE
    assert L.sp24_splitk_workspace_bytes(64, 64, 509, sp24.BF16) == 0
