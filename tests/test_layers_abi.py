"""Host-only checks of the operators around the products: every refusal comes before a device is touched (the addresses are made up)."""
import ctypes

import pytest

from paper_2104_08378_amd import sp24

OK, NULL, SHAPE, ALIGN, DTYPE, LAYOUT = 0, 1, 2, 3, 4, 5
STEP = 0x10000000
A, B, C, D, E, F, G, W = (STEP * i for i in range(1, 9))       # fake, aligned, far apart
f = ctypes.c_float


def norm(X=A, R=B, w=C, eps=1e-6, Y=D, sc=E, h=F, rs=G, N=8, H=64, ldx=64, ldr=64, ldy=64, ldh=64, t=sp24.BF16, out=sp24.I8):
    return sp24.lib().sp24_rmsnorm(X, R, w, f(eps), Y, sc, h, rs, N, H, ldx, ldr, ldy, ldh, t, out, None)


@pytest.mark.parametrize("bad,want", [
    (dict(X=0), NULL), (dict(w=0), NULL), (dict(Y=0), NULL), (dict(sc=0), NULL), (dict(ldx=63), SHAPE), (dict(ldr=63), SHAPE), (dict(ldy=63), SHAPE),
    (dict(ldh=63), SHAPE), (dict(H=0), SHAPE), (dict(H=32769, ldx=40000, ldr=40000, ldy=40000, ldh=40000), SHAPE), (dict(N=-1), SHAPE), (dict(eps=-1.0), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(X=A + 1), ALIGN), (dict(w=C + 2), ALIGN), (dict(rs=G + 1), ALIGN), (dict(sc=E + 3), ALIGN), (dict(t=sp24.I8), DTYPE),
    (dict(out=sp24.I32), DTYPE), (dict(Y=F), SHAPE), (dict(Y=A), SHAPE), (dict(h=A, ldh=72), SHAPE), (dict(h=A + 64), SHAPE), (dict(sc=B), SHAPE), (dict(rs=E), SHAPE),
    (dict(h=C), SHAPE), (dict(N=0, X=0, Y=0, w=0), OK)])
def test_norm(bad, want):
    assert norm(**bad) == want


def test_quantisation_and_norm_gradient():
    L = sp24.lib()
    q = lambda X=A, Q=B, sc=C, N=8, H=64, ldx=64, ldq=64, t=sp24.F16, out=sp24.F8: L.sp24_quantize_rows(X, Q, sc, N, H, ldx, ldq, t, out, None)  # noqa: E731
    assert q(X=0) == NULL and q(sc=0) == NULL and q(H=65537, ldx=70000, ldq=70000) == SHAPE and q(out=sp24.BF16) == DTYPE and q(t=sp24.F8) == DTYPE
    assert q(Q=A) == SHAPE and q(ldq=60) == SHAPE and q(X=A + 1) == ALIGN and q(N=0) == OK
    need = L.sp24_rmsnorm_backward_workspace_bytes(8, 64)
    assert need >= 64 * 4 and L.sp24_rmsnorm_backward_workspace_bytes(0, 64) == 0 and L.sp24_rmsnorm_backward_workspace_bytes(8, 0) == 0

    def grad(dY=A, h=B, w=C, rs=D, dh=E, dX=F, dw=G, N=8, H=64, ld=64, t=sp24.BF16, ws=W, bytes=need):
        return L.sp24_rmsnorm_backward(dY, h, w, rs, dh, dX, dw, N, H, ld, 64, 64, 64, t, ws, bytes, None)
    assert grad(dY=0) == NULL and grad(h=0) == NULL and grad(rs=0) == NULL and grad(dw=0) == NULL and grad(ws=0) == NULL and grad(dX=0) == NULL
    assert grad(bytes=need - 1) == SHAPE and grad(ws=W + 8) == ALIGN and grad(ld=60) == SHAPE and grad(t=sp24.I8) == DTYPE
    assert grad(dX=A + 128) == SHAPE and grad(dw=B) == SHAPE and grad(ws=A) == SHAPE and grad(dX=C) == SHAPE


def linear(V=A, mt=B, X=C, Y=D, M=64, N=16, K=64, ldx=64, ldy=64, ws=0, xs=0, b=0, act=0, r=0, ldr=64, z=0, ldz=64, i=sp24.BF16, o=sp24.BF16, l=1):
    return sp24.lib().sp24_linear(V, mt, X, Y, M, N, K, ldx, ldy, ws, xs, b, act, r, ldr, z, ldz, i, o, l, None)


@pytest.mark.parametrize("bad,want", [
    (dict(V=0), NULL), (dict(mt=0), NULL), (dict(X=0), NULL), (dict(Y=0), NULL), (dict(M=48), LAYOUT), (dict(l=7), LAYOUT), (dict(K=72, ldx=72), SHAPE),
    (dict(ldx=32), SHAPE), (dict(ldy=32), SHAPE), (dict(r=E, ldr=32), SHAPE), (dict(z=E, ldz=32), SHAPE), (dict(N=-1), SHAPE), (dict(M=-32), SHAPE),
    (dict(V=A + 8), ALIGN), (dict(mt=B + 4), ALIGN), (dict(X=C + 1), ALIGN), (dict(b=E + 2), ALIGN), (dict(act=4), DTYPE), (dict(act=-1), DTYPE),
    (dict(o=sp24.I8), DTYPE), (dict(i=sp24.F32), DTYPE), (dict(ws=E), DTYPE), (dict(xs=E), DTYPE), (dict(Y=C), SHAPE), (dict(z=D), SHAPE), (dict(r=D + 128), SHAPE),
    (dict(r=D, ldr=72), SHAPE), (dict(b=D), SHAPE), (dict(i=sp24.I8, ws=D), SHAPE), (dict(i=sp24.I8, K=32, ldx=32, l=0, xs=D + 64), SHAPE), (dict(N=0, X=0, Y=0), OK),
    (dict(M=0), OK)])
def test_linear(bad, want):
    assert linear(**bad) == want


def test_experts():
    L = sp24.lib()

    def grouped(V=A, mt=B, X=C, Y=D, of=E, n=4, M=64, R=32, K=64, b=0, i=sp24.BF16, l=1):
        return L.sp24_linear_grouped(V, mt, X, Y, of, n, M, R, K, K, M, 0, 0, b, 0, 0, 0, i, sp24.BF16, l, None)
    assert grouped(of=0) == NULL and grouped(of=E + 2) == ALIGN and grouped(n=0) == SHAPE and grouped(n=1025) == SHAPE and grouped(R=24) == SHAPE
    assert grouped(Y=E) == SHAPE and grouped(V=0) == NULL and grouped(M=40) == LAYOUT and grouped(b=D) == SHAPE and grouped(R=0) == OK
    assert grouped(Y=A + 3 * 64 * 32 * 2) == SHAPE                     # the last expert's values

    def dense(Aa=A, Bb=B, Dd=D, of=E, n=4, M=64, N=64, R=32, lda=32, ldb=64, ldd=64, i=sp24.BF16, o=sp24.F32):
        return L.sp24_gemm_dense_grouped(Aa, Bb, Dd, of, n, M, N, R, lda, ldb, ldd, i, o, None)
    assert dense(Aa=0) == NULL and dense(of=0) == NULL and dense(lda=24) == SHAPE and dense(lda=36) == ALIGN and dense(N=60) == SHAPE and dense(R=40) == SHAPE
    assert dense(i=sp24.I8) == DTYPE and dense(o=sp24.F16) == DTYPE and dense(Dd=B) == SHAPE and dense(ldb=1 << 21) == SHAPE and dense(M=0) == OK
    need = L.sp24_linear_backward_workspace_bytes(64, 32, 1)
    assert need == 2 * 64 * 4 and L.sp24_linear_backward_workspace_bytes(64, 65, 0) == 2 * 64 * 4

    def back(dY=A, Z=B, dZ=C, dZt=D, db=E, M=64, N=32, ld=64, ldt=32, act=2, of=F, n=4, t=sp24.F16, ws=G, bytes=need):
        return L.sp24_linear_backward(dY, Z, dZ, dZt, db, M, N, ld, 64, 64, ldt, act, of, n, t, ws, bytes, None)
    assert back(dY=0) == NULL and back(Z=0) == NULL and back(ws=0) == NULL and back(bytes=need - 4) == SHAPE and back(N=24, ldt=24) == SHAPE
    assert back(act=9) == DTYPE and back(t=sp24.F32) == DTYPE and back(ldt=31) == SHAPE and back(ld=63) == SHAPE and back(n=0) == SHAPE and back(of=F + 1) == ALIGN
    assert back(dZt=A) == SHAPE and back(dZ=A + 2) == SHAPE and back(db=G) == SHAPE and back(dZ=D) == SHAPE and back(M=0) == OK


def test_sort_gather_and_combine():
    L = sp24.lib()
    assert [sp24.sp24_moe_rows(t, e) for t, e in ((0, 8), (1, 8), (16, 1), (17, 1), (32, 8), (100, 1024))] == [0, 16, 16 + 0 * 1, 32, 144, 1600]
    assert sp24.sp24_moe_rows(-1, 8) == 0 and sp24.sp24_moe_rows(8, 0) == 0 and sp24.sp24_moe_rows(8, 1025) == 0
    assert L.sp24_moe_sort_workspace_bytes(1 << 17, 8) == 0 and L.sp24_moe_sort_workspace_bytes((1 << 17) + 1, 8) == 9 * 8 * 4

    def sort(ids=A, of=B, sl=C, ro=D, T=100, n=8, R=220, ws=0, bytes=0):
        return L.sp24_moe_sort(ids, of, sl, ro, T, n, R, ws, bytes, None)
    assert sort(ids=0) == NULL and sort(of=0) == NULL and sort(sl=0) == NULL and sort(ro=0) == NULL and sort(R=200) == SHAPE and sort(n=0) == SHAPE and sort(T=-1) == SHAPE
    assert sort(ids=A + 2) == ALIGN and sort(sl=A) == SHAPE and sort(ro=B) == SHAPE and sort(T=200000, R=201000) == NULL and sort(T=200000, R=201000, ws=E, bytes=32) == SHAPE

    def gather(X=A, sc=0, ro=B, Xs=C, so=0, N=8, R=32, k=2, H=64, ldx=64, ldxs=64, t=sp24.I8):
        return L.sp24_moe_gather(X, sc, ro, Xs, so, N, R, k, H, ldx, ldxs, t, None)
    assert gather(X=0) == NULL and gather(ro=0) == NULL and gather(Xs=0) == NULL and gather(sc=D) == NULL and gather(k=0) == SHAPE and gather(H=0) == SHAPE
    assert gather(ldx=60) == SHAPE and gather(t=sp24.I32) == DTYPE and gather(Xs=A) == SHAPE and gather(sc=D, so=C) == SHAPE and gather(R=0) == OK

    def combine(Y=A, sl=B, w=C, r=D, o=E, N=8, R=32, k=2, H=64, ldy=64, ldr=64, ldo=64, t=sp24.BF16):
        return L.sp24_moe_combine(Y, sl, w, r, o, N, R, k, H, ldy, ldr, ldo, t, None)
    assert combine(Y=0) == NULL and combine(sl=0) == NULL and combine(o=0) == NULL and combine(o=A) == SHAPE and combine(o=D + 128) == SHAPE and combine(ldo=60) == SHAPE
    assert combine(t=sp24.I8) == DTYPE and combine(o=E + 1) == ALIGN and combine(w=C + 1) == ALIGN and combine(k=0) == SHAPE and combine(N=0) == OK

    def back(d=A, Y=B, ro=C, sl=D, w=E, dY=F, dw=G, N=8, R=32, k=2, H=64, t=sp24.BF16):
        return L.sp24_moe_combine_backward(d, Y, ro, sl, w, dY, dw, N, R, k, H, H, H, H, t, None)
    assert back(d=0) == NULL and back(Y=0) == NULL and back(ro=0) == NULL and back(sl=0) == NULL and back(w=0) == NULL and back(dY=0) == NULL and back(dw=0) == NULL
    assert back(dY=A) == SHAPE and back(dw=E) == SHAPE and back(t=sp24.F8) == DTYPE and back(dY=B + 128) == SHAPE and back(k=0) == SHAPE
