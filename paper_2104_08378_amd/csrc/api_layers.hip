// C ABI of the operators around the products: argument validation on the host, then the launch.
#include <cmath>
#include <initializer_list>

#include "checks.hpp"
#include "launch.hpp"
#include "linear.hpp"

using namespace sp24;

namespace {

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 64, kMostMm = (int64_t)1 << 30, kMostNorm = 32768, kMostQuantised = 65536;

bool is_float16(sp24_dtype t) { return t == SP24_F16 || t == SP24_BF16; }
bool is_float(sp24_dtype t) { return is_float16(t) || t == SP24_F32; }
bool is_code(sp24_dtype t) { return t == SP24_I8 || t == SP24_F8; }
bool is_act(sp24_act a) { return a == SP24_ACT_NONE || a == SP24_ACT_RELU || a == SP24_ACT_GELU || a == SP24_ACT_SILU; }
bool misaligned(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }

// a buffer of a call: its first byte and the bytes it spans (0: not there)
struct Span {
    const void* p;
    size_t bytes;
};
Span matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int es)
{
    return {p, p && rows > 0 && cols > 0 ? ((size_t)(rows - 1) * ld + cols) * es : 0};
}
Span vec(const void* p, int64_t n, int es) { return {p, p && n > 0 ? (size_t)n * es : 0}; }

// does `out` share bytes with one of `others`?  (Ranges from the first element's byte to the last's: rows that lie between another buffer's rows count)
bool overlaps(Span out, std::initializer_list<Span> others)
{
    for (const Span& o : others)
        if (out.bytes != 0 && o.bytes != 0 && ranges_overlap(out.p, out.bytes, o.p, o.bytes)) return true;
    return false;
}
// in place: the same first byte and the same row pitch
bool in_place(Span out, int64_t ld, Span in, int64_t ld_in, int es, int es_in) { return out.p == in.p && es == es_in && ld == ld_in; }

#define SP24_TRY(expr)                    \
    do {                                  \
        const sp24_status s_ = (expr);    \
        if (s_ != SP24_OK) return s_;     \
    } while (0)

sp24_status check_vector(const void* p, int size = 4)
{
    if (!p) return SP24_ERR_NULL;
    return misaligned(p, size) ? SP24_ERR_ALIGN : SP24_OK;
}

int64_t segment_rows(int64_t T, int experts)
{
    return (T + (kSegmentRows - 1) * std::min<int64_t>(T, experts)) / kSegmentRows * kSegmentRows;
}

} // namespace

extern "C" {

sp24_status sp24_rmsnorm(const void* X, const void* residual, const float* weight, float eps, void* Y, float* scale, void* hidden, float* rstd,
                         int64_t N, int64_t H, int64_t ldx, int64_t ldr, int64_t ldy, int64_t ldh, sp24_dtype t, sp24_dtype out, void* stream)
{
    if (!is_float(t) || !(is_float(out) || is_code(out))) return SP24_ERR_DTYPE;
    if (N < 0 || H < 1 || N > kMostRows || H > kMostNorm || !(eps >= 0.0f) || std::isinf(eps)) return SP24_ERR_SHAPE;
    if (N == 0) return SP24_OK;
    const int es = esize_of(t), os = esize_of(out);
    SP24_TRY(check_matrix(X, N, H, ldx, es, false));
    SP24_TRY(check_matrix(Y, N, H, ldy, os, false));
    if (residual) SP24_TRY(check_matrix(residual, N, H, ldr, es, false));
    if (hidden) SP24_TRY(check_matrix(hidden, N, H, ldh, es, false));
    SP24_TRY(check_vector(weight));
    if (is_code(out)) SP24_TRY(check_vector(scale));
    if (rstd) SP24_TRY(check_vector(rstd));
    const Span x = matrix(X, N, H, ldx, es), r = matrix(residual, N, H, ldr, es), y = matrix(Y, N, H, ldy, os), h = matrix(hidden, N, H, ldh, es),
               w = vec(weight, H, 4), sc = vec(is_code(out) ? scale : nullptr, N, 4), rs = vec(rstd, N, 4);
    if (overlaps(y, {h, w, sc, rs}) || overlaps(h, {w, sc, rs}) || overlaps(sc, {x, r, w, rs}) || overlaps(rs, {x, r, w})) return SP24_ERR_SHAPE;
    for (const Span* in : {&x, &r}) {
        const int64_t ld = in == &x ? ldx : ldr;
        if (overlaps(y, {*in}) && !in_place(y, ldy, *in, ld, os, es)) return SP24_ERR_SHAPE;
        if (overlaps(h, {*in}) && !in_place(h, ldh, *in, ld, es, es)) return SP24_ERR_SHAPE;
    }
    return launch_norm_rows(RowsArgs{X, residual, weight, Y, hidden, scale, rstd, N, H, ldx, ldr, ldy, ldh, eps, t, out}, static_cast<hipStream_t>(stream));
}

sp24_status sp24_quantize_rows(const void* X, void* Q, float* scale, int64_t N, int64_t H, int64_t ldx, int64_t ldq, sp24_dtype t, sp24_dtype out,
                               void* stream)
{
    if (!is_float(t) || !is_code(out)) return SP24_ERR_DTYPE;
    if (N < 0 || H < 1 || N > kMostRows || H > kMostQuantised) return SP24_ERR_SHAPE;
    if (N == 0) return SP24_OK;
    const int es = esize_of(t);
    SP24_TRY(check_matrix(X, N, H, ldx, es, false));
    SP24_TRY(check_matrix(Q, N, H, ldq, 1, false));
    SP24_TRY(check_vector(scale));
    const Span x = matrix(X, N, H, ldx, es), q = matrix(Q, N, H, ldq, 1), sc = vec(scale, N, 4);
    if (overlaps(q, {x, sc}) || overlaps(sc, {x})) return SP24_ERR_SHAPE;
    return launch_norm_rows(RowsArgs{X, nullptr, nullptr, Q, nullptr, scale, nullptr, N, H, ldx, 0, ldq, 0, 0.0f, t, out}, static_cast<hipStream_t>(stream));
}

size_t sp24_rmsnorm_backward_workspace_bytes(int64_t N, int64_t H)
{
    if (N < 0 || H < 1 || N > kMostRows || H > kMostNorm) return 0;
    return (size_t)norm_grad_groups(N, H) * H * 4;
}

sp24_status sp24_rmsnorm_backward(const void* dY, const void* hidden, const float* weight, const float* rstd, const void* dhidden, void* dX,
                                  float* dweight, int64_t N, int64_t H, int64_t lddy, int64_t ldh, int64_t lddh, int64_t lddx, sp24_dtype t,
                                  void* workspace, size_t workspace_bytes, void* stream)
{
    if (!is_float(t)) return SP24_ERR_DTYPE;
    if (N < 0 || H < 1 || N > kMostRows || H > kMostNorm) return SP24_ERR_SHAPE;
    const int es = esize_of(t);
    SP24_TRY(check_vector(weight));
    SP24_TRY(check_vector(dweight));
    const size_t need = sp24_rmsnorm_backward_workspace_bytes(N, H);
    if (N > 0) {
        SP24_TRY(check_matrix(dY, N, H, lddy, es, false));
        SP24_TRY(check_matrix(hidden, N, H, ldh, es, false));
        SP24_TRY(check_matrix(dX, N, H, lddx, es, false));
        if (dhidden) SP24_TRY(check_matrix(dhidden, N, H, lddh, es, false));
        SP24_TRY(check_vector(rstd));
        if (!workspace) return SP24_ERR_NULL;
        if (!aligned16(workspace)) return SP24_ERR_ALIGN;
        if (workspace_bytes < need) return SP24_ERR_SHAPE;
    }
    const Span dy = matrix(dY, N, H, lddy, es), h = matrix(hidden, N, H, ldh, es), dh = matrix(dhidden, N, H, lddh, es), dx = matrix(dX, N, H, lddx, es),
               w = vec(weight, H, 4), rs = vec(rstd, N, 4), dw = vec(dweight, H, 4), ws = Span{workspace, need};
    if (overlaps(dx, {w, rs, dw, ws}) || overlaps(dw, {dy, h, dh, w, rs, ws}) || overlaps(ws, {dy, h, dh, w, rs})) return SP24_ERR_SHAPE;
    if ((overlaps(dx, {dy}) && !in_place(dx, lddx, dy, lddy, es, es)) || (overlaps(dx, {h}) && !in_place(dx, lddx, h, ldh, es, es)) ||
        (overlaps(dx, {dh}) && !in_place(dx, lddx, dh, lddh, es, es)))
        return SP24_ERR_SHAPE;
    return launch_norm_grad(NormGradArgs{dY, hidden, dhidden, weight, rstd, dX, static_cast<float*>(workspace), dweight, N, H, lddy, ldh, lddh, lddx, t},
                            static_cast<hipStream_t>(stream));
}

// What both layer entry points check.  rows: of X and Y; weight_rows: M, or those of all experts
static sp24_status check_linear(const LinearArgs& a, int64_t rows, int64_t weight_rows, const void* offsets, int experts)
{
    const int es = esize_of(a.in), os = esize_of(a.out);
    if (!is_input_type(a.in) || !is_float(a.out)) return SP24_ERR_DTYPE;
    if (!is_act((sp24_act)a.act)) return SP24_ERR_DTYPE;
    if (!is_layout(a.layout)) return SP24_ERR_LAYOUT;
    if (a.M < 0 || rows < 0 || rows > kMostMm || a.M > kMostMm || a.K > kMostMm || !k_legal(a.K, a.in)) return SP24_ERR_SHAPE;
    if (!layout_fits(a.M, a.K, a.layout)) return SP24_ERR_LAYOUT;
    if (!is_code(a.in) && (a.epi.w_scale || a.x_scale)) return SP24_ERR_DTYPE;
    if (a.M == 0 || rows == 0) return SP24_OK;
    if (((a.M + 31) / 32) * (rows / 16 + 2) >= ((int64_t)1 << 31)) return SP24_ERR_SHAPE;
    if (!a.A || !a.meta) return SP24_ERR_NULL;
    if (!aligned16(a.A) || !aligned16(a.meta)) return SP24_ERR_ALIGN;
    SP24_TRY(check_matrix(a.B, rows, a.K, a.ldb, es, false));
    SP24_TRY(check_matrix(a.D, rows, a.M, a.ldd, os, false));
    if (a.residual) SP24_TRY(check_matrix(a.residual, rows, a.M, a.ldr, os, false));
    if (a.Z) SP24_TRY(check_matrix(a.Z, rows, a.M, a.ldz, os, false));
    if (misaligned(a.epi.w_scale, 4) || misaligned(a.x_scale, 4) || misaligned(a.epi.bias, 4)) return SP24_ERR_ALIGN;
    const Span v = {a.A, (size_t)weight_rows * (a.K / 2) * es}, mt = {a.meta, (size_t)weight_rows * (a.K / 8)}, x = matrix(a.B, rows, a.K, a.ldb, es),
               y = matrix(a.D, rows, a.M, a.ldd, os), r = matrix(a.residual, rows, a.M, a.ldr, os), z = matrix(a.Z, rows, a.M, a.ldz, os),
               ws = vec(a.epi.w_scale, weight_rows, 4), xs = vec(a.x_scale, rows, 4), b = vec(a.epi.bias, weight_rows, 4),
               of = vec(offsets, offsets ? experts + 1 : 0, 4);
    if (overlaps(y, {v, mt, x, z, ws, xs, b, of}) || overlaps(z, {v, mt, x, r, ws, xs, b, of})) return SP24_ERR_SHAPE;
    if (overlaps(y, {r}) && !in_place(y, a.ldd, r, a.ldr, os, os)) return SP24_ERR_SHAPE;
    return SP24_OK;
}

static void set_linear(LinearArgs& a, const void* V, const void* meta, const void* X, void* Y, int64_t M, int64_t N, int64_t K, int64_t ldx,
                       int64_t ldy, const float* w_scale, const float* x_scale, const float* bias, sp24_act act, sp24_dtype in, sp24_dtype out,
                       sp24_layout l)
{
    static_cast<MmArgs&>(a) = MmArgs{V, meta, X, Y, M, N, K, 0, ldx, ldy, in, out, SP24_B_KMAJOR, l, true};
    a.epi.w_scale = w_scale;
    a.epi.bias = bias;
    a.x_scale = x_scale;
    a.act = act;
}

sp24_status sp24_linear(const void* V, const void* meta, const void* X, void* Y, int64_t M, int64_t N, int64_t K, int64_t ldx, int64_t ldy,
                        const float* w_scale, const float* x_scale, const float* bias, sp24_act act, const void* residual, int64_t ldr, void* Z,
                        int64_t ldz, sp24_dtype in, sp24_dtype out, sp24_layout l, void* stream)
{
    LinearArgs a{};
    set_linear(a, V, meta, X, Y, M, N, K, ldx, ldy, w_scale, x_scale, bias, act, in, out, l);
    a.residual = residual;
    a.ldr = ldr;
    a.Z = Z;
    a.ldz = ldz;
    SP24_TRY(check_linear(a, N, M, nullptr, 0));
    return M == 0 || N == 0 ? SP24_OK : launch_linear(a, static_cast<hipStream_t>(stream));
}

sp24_status sp24_linear_grouped(const void* V, const void* meta, const void* X, void* Y, const int32_t* offsets, int experts, int64_t M, int64_t rows,
                                int64_t K, int64_t ldx, int64_t ldy, const float* w_scale, const float* x_scale, const float* bias, sp24_act act,
                                void* Z, int64_t ldz, sp24_dtype in, sp24_dtype out, sp24_layout l, void* stream)
{
    GroupedArgs a{};
    set_linear(a, V, meta, X, Y, M, rows, K, ldx, ldy, w_scale, x_scale, bias, act, in, out, l);
    a.Z = Z;
    a.ldz = ldz;
    a.offsets = offsets;
    a.experts = experts;
    if (experts < 1 || experts > SP24_MOST_EXPERTS || rows % kSegmentRows != 0) return SP24_ERR_SHAPE;
    SP24_TRY(check_linear(a, rows, M * experts, offsets, experts));
    if (M == 0 || rows == 0) return SP24_OK;
    SP24_TRY(check_vector(offsets));
    return launch_linear_grouped(a, static_cast<hipStream_t>(stream));
}

sp24_status sp24_gemm_dense_grouped(const void* A, const void* B, void* D, const int32_t* offsets, int experts, int64_t M, int64_t N, int64_t rows,
                                    int64_t lda, int64_t ldb, int64_t ldd, sp24_dtype in, sp24_dtype out, void* stream)
{
    if (!is_float16(in) || !(out == SP24_F32 || out == in)) return SP24_ERR_DTYPE;
    if (M < 0 || N < 0 || N % 8 != 0 || rows < 0 || rows > kMostRows || rows % kSegmentRows != 0 || experts < 1 || experts > SP24_MOST_EXPERTS)
        return SP24_ERR_SHAPE;
    if (M > kMostRows || N > kMostRows || ((M + 127) / 128) * ((N + 127) / 128) >= ((int64_t)1 << 31)) return SP24_ERR_SHAPE;
    if (lda * 2 >= ((int64_t)1 << 22) || ldb * 2 >= ((int64_t)1 << 22)) return SP24_ERR_SHAPE;      // 32-bit offsets inside a tile
    if (M == 0 || N == 0) return SP24_OK;
    SP24_TRY(check_vector(offsets));
    const int os = esize_of(out);
    if (rows > 0) {
        SP24_TRY(check_matrix(A, M, rows, lda, 2));
        SP24_TRY(check_matrix(B, rows, N, ldb, 2));
    }
    SP24_TRY(check_matrix(D, (int64_t)experts * M, N, ldd, os, false));
    const Span d = matrix(D, (int64_t)experts * M, N, ldd, os);
    if (overlaps(d, {matrix(A, M, rows, lda, 2), matrix(B, rows, N, ldb, 2), vec(offsets, experts + 1, 4)})) return SP24_ERR_SHAPE;
    SegmentArgs a{};
    static_cast<MmArgs&>(a) = MmArgs{A, nullptr, B, D, M, N, rows, lda, ldb, ldd, in, out, SP24_B_NMAJOR, SP24_LAYOUT_CANONICAL, false};
    a.offsets = offsets;
    return launch_gemm_grouped(a, experts, static_cast<hipStream_t>(stream));
}

static int grad_unit(const int32_t* offsets) { return offsets ? kSegmentRows : 64; }

size_t sp24_linear_backward_workspace_bytes(int64_t M, int64_t N, int grouped)
{
    if (M < 0 || N < 0 || N > kMostRows || M > kMostRows) return 0;
    const int unit = grouped ? kSegmentRows : 64;
    return (size_t)((N + unit - 1) / unit) * M * 4;
}

sp24_status sp24_linear_backward(const void* dY, const void* Z, void* dZ, void* dZt, float* dbias, int64_t M, int64_t N, int64_t lddy, int64_t ldz,
                                 int64_t lddz, int64_t lddzt, sp24_act act, const int32_t* offsets, int experts, sp24_dtype t, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    if (!is_float16(t) || !is_act(act)) return SP24_ERR_DTYPE;
    if (M < 0 || N < 0 || M > kMostRows || N > kMostRows || ((M + 63) / 64) * ((N + 63) / 64) >= ((int64_t)1 << 31)) return SP24_ERR_SHAPE;
    if (offsets && (experts < 1 || experts > SP24_MOST_EXPERTS || N % kSegmentRows != 0)) return SP24_ERR_SHAPE;
    if (offsets && misaligned(offsets, 4)) return SP24_ERR_ALIGN;
    if (M == 0) return SP24_OK;
    SP24_TRY(check_matrix(dY, N, M, lddy, 2, false));
    if (act != SP24_ACT_NONE) SP24_TRY(check_matrix(Z, N, M, ldz, 2, false));
    if (dZ) SP24_TRY(check_matrix(dZ, N, M, lddz, 2, false));
    if (dZt && N > 0) SP24_TRY(check_matrix(dZt, M, N, lddzt, 2, false));
    const size_t need = dbias ? sp24_linear_backward_workspace_bytes(M, N, offsets != nullptr) : 0;
    if (dbias) {
        SP24_TRY(check_vector(dbias));
        if (need > 0 && !workspace) return SP24_ERR_NULL;
        if (need > 0 && !aligned16(workspace)) return SP24_ERR_ALIGN;
        if (workspace_bytes < need) return SP24_ERR_SHAPE;
    }
    const Span dy = matrix(dY, N, M, lddy, 2), z = matrix(act != SP24_ACT_NONE ? Z : nullptr, N, M, ldz, 2), dz = matrix(dZ, N, M, lddz, 2),
               dzt = matrix(dZt, M, N, lddzt, 2), db = vec(dbias, (offsets ? experts : 1) * M, 4), ws = Span{workspace, need},
               of = vec(offsets, offsets ? experts + 1 : 0, 4);
    if (overlaps(dz, {dzt, db, ws, of}) || overlaps(dzt, {dy, z, db, ws, of}) || overlaps(db, {dy, z, ws, of}) || overlaps(ws, {dy, z, of})) return SP24_ERR_SHAPE;
    if ((overlaps(dz, {dy}) && !in_place(dz, lddz, dy, lddy, 2, 2)) || (overlaps(dz, {z}) && !in_place(dz, lddz, z, ldz, 2, 2))) return SP24_ERR_SHAPE;
    return launch_linear_grad(LinearGradArgs{dY, Z, dZ, dZt, dbias ? static_cast<float*>(workspace) : nullptr, dbias, offsets, M, N, lddy, ldz, lddz, lddzt,
                                             (int)act, experts, grad_unit(offsets), t},
                              static_cast<hipStream_t>(stream));
}

int64_t sp24_moe_rows(int64_t choices, int experts)
{
    if (choices < 0 || choices > kMostRows / 16 || experts < 1 || experts > SP24_MOST_EXPERTS) return 0;
    return segment_rows(choices, experts);
}

size_t sp24_moe_sort_workspace_bytes(int64_t choices, int experts)
{
    if (choices <= kSortAtOnce || choices > kMostRows / 16 || experts < 1 || experts > SP24_MOST_EXPERTS) return 0;
    return (size_t)((choices + kSortPart - 1) / kSortPart) * experts * 4;
}

sp24_status sp24_moe_sort(const int32_t* ids, int32_t* offsets, int32_t* slots, int32_t* rows, int64_t choices, int experts, int64_t row_count,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    if (choices < 0 || choices > kMostRows / 16 || experts < 1 || experts > SP24_MOST_EXPERTS) return SP24_ERR_SHAPE;
    if (row_count < segment_rows(choices, experts) || row_count > kMostRows) return SP24_ERR_SHAPE;
    SP24_TRY(check_vector(offsets));
    if (choices > 0) {
        SP24_TRY(check_vector(ids));
        SP24_TRY(check_vector(slots));
    }
    if (row_count > 0) SP24_TRY(check_vector(rows));
    const size_t need = sp24_moe_sort_workspace_bytes(choices, experts);
    if (need > 0) {
        if (!workspace) return SP24_ERR_NULL;
        if (misaligned(workspace, 4)) return SP24_ERR_ALIGN;
        if (workspace_bytes < need) return SP24_ERR_SHAPE;
    }
    const Span id = vec(ids, choices, 4), of = vec(offsets, experts + 1, 4), sl = vec(slots, choices, 4), ro = vec(rows, row_count, 4), ws = Span{workspace, need};
    if (overlaps(of, {id, sl, ro, ws}) || overlaps(sl, {id, ro, ws}) || overlaps(ro, {id, ws}) || overlaps(ws, {id})) return SP24_ERR_SHAPE;
    return launch_moe_sort(SortArgs{ids, offsets, slots, rows, static_cast<int32_t*>(workspace), choices, row_count, experts}, static_cast<hipStream_t>(stream));
}

sp24_status sp24_moe_gather(const void* X, const float* scale, const int32_t* rows, void* Xs, float* scale_out, int64_t N, int64_t row_count, int topk,
                            int64_t H, int64_t ldx, int64_t ldxs, sp24_dtype t, void* stream)
{
    if (!(is_float(t) || is_code(t))) return SP24_ERR_DTYPE;
    if (N < 0 || row_count < 0 || N > kMostRows || row_count > kMostRows || topk < 1 || H < 1 || H > kMostRows) return SP24_ERR_SHAPE;
    if (row_count == 0) return SP24_OK;
    const int es = esize_of(t);
    if (row_count * ((H * es + 4095) / 4096) >= ((int64_t)1 << 31)) return SP24_ERR_SHAPE;
    SP24_TRY(check_matrix(X, N, H, ldx, es, false));
    SP24_TRY(check_matrix(Xs, row_count, H, ldxs, es, false));
    SP24_TRY(check_vector(rows));
    if (scale || scale_out) {
        if (N > 0) SP24_TRY(check_vector(scale));               // (no tokens: no choice has one, and the scales are zeros)
        SP24_TRY(check_vector(scale_out));
    }
    const Span x = matrix(X, N, H, ldx, es), xs = matrix(Xs, row_count, H, ldxs, es), ro = vec(rows, row_count, 4), sc = vec(scale, N, 4),
               so = vec(scale_out, row_count, 4);
    if (overlaps(xs, {x, ro, sc, so}) || overlaps(so, {x, ro, sc})) return SP24_ERR_SHAPE;
    return launch_moe_gather(GatherArgs{X, scale, rows, Xs, scale_out, N, row_count, H * es, ldx * es, ldxs * es, topk}, static_cast<hipStream_t>(stream));
}

sp24_status sp24_moe_combine(const void* Y, const int32_t* slots, const float* weights, const void* residual, void* out, int64_t N, int64_t row_count,
                             int topk, int64_t H, int64_t ldy, int64_t ldr, int64_t ldo, sp24_dtype t, void* stream)
{
    if (!is_float(t)) return SP24_ERR_DTYPE;
    if (N < 0 || row_count < 0 || N > kMostRows || row_count > kMostRows || topk < 1 || H < 1 || H > kMostRows) return SP24_ERR_SHAPE;
    if (N == 0) return SP24_OK;
    if (N * ((H + 2047) / 2048) >= ((int64_t)1 << 31) || topk > kMostRows / N) return SP24_ERR_SHAPE;
    const int es = esize_of(t);
    SP24_TRY(check_matrix(Y, row_count, H, ldy, es, false));
    SP24_TRY(check_matrix(out, N, H, ldo, es, false));
    if (residual) SP24_TRY(check_matrix(residual, N, H, ldr, es, false));
    SP24_TRY(check_vector(slots));
    if (weights) SP24_TRY(check_vector(weights));
    const Span y = matrix(Y, row_count, H, ldy, es), o = matrix(out, N, H, ldo, es), r = matrix(residual, N, H, ldr, es), sl = vec(slots, N * topk, 4),
               w = vec(weights, N * topk, 4);
    if (overlaps(o, {y, sl, w}) || (overlaps(o, {r}) && !in_place(o, ldo, r, ldr, es, es))) return SP24_ERR_SHAPE;
    return launch_moe_combine(CombineArgs{Y, residual, slots, weights, out, N, row_count, H, ldy, ldr, ldo, topk, t}, static_cast<hipStream_t>(stream));
}

sp24_status sp24_moe_combine_backward(const void* dOut, const void* Y, const int32_t* rows, const int32_t* slots, const float* weights, void* dY,
                                      float* dweights, int64_t N, int64_t row_count, int topk, int64_t H, int64_t lddo, int64_t ldy, int64_t lddy,
                                      sp24_dtype t, void* stream)
{
    if (!is_float(t)) return SP24_ERR_DTYPE;
    if (N < 0 || row_count < 0 || N > kMostRows || row_count > kMostRows || topk < 1 || H < 1 || H > kMostRows) return SP24_ERR_SHAPE;
    if (N == 0 && row_count == 0) return SP24_OK;
    if (N > 0 && topk > kMostRows / N) return SP24_ERR_SHAPE;
    const int es = esize_of(t);
    SP24_TRY(check_matrix(dOut, N, H, lddo, es, false));
    SP24_TRY(check_matrix(Y, row_count, H, ldy, es, false));
    SP24_TRY(check_matrix(dY, row_count, H, lddy, es, false));
    if (N > 0) {
        SP24_TRY(check_vector(slots));
        SP24_TRY(check_vector(weights));
        SP24_TRY(check_vector(dweights));
    }
    if (row_count > 0) SP24_TRY(check_vector(rows));
    const Span d = matrix(dOut, N, H, lddo, es), y = matrix(Y, row_count, H, ldy, es), dy = matrix(dY, row_count, H, lddy, es), ro = vec(rows, row_count, 4),
               sl = vec(slots, N * topk, 4), w = vec(weights, N * topk, 4), dw = vec(dweights, N * topk, 4);
    if (overlaps(dy, {d, ro, sl, w, dw}) || overlaps(dw, {d, y, ro, sl, w})) return SP24_ERR_SHAPE;
    if (overlaps(dy, {y}) && !in_place(dy, lddy, y, ldy, es, es)) return SP24_ERR_SHAPE;
    return launch_moe_combine_grad(CombineGradArgs{dOut, Y, rows, slots, weights, dY, dweights, N, row_count, H, lddo, ldy, lddy, topk, t},
                                   static_cast<hipStream_t>(stream));
}

} // extern "C"
