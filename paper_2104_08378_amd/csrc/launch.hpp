// Internal launch entry points shared by the C-ABI layer (api.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/sp24.h"
#include "common.hpp"

namespace sp24 {

sp24_status launch_prune(const void* A, void* P, int64_t M, int64_t K, int64_t lda, int64_t ldp, sp24_dtype t, hipStream_t st);
sp24_status launch_compress(const void* A, void* V, void* meta, int64_t M, int64_t K, int64_t lda, sp24_dtype t, sp24_layout l, hipStream_t st);
sp24_status launch_prune_transposable(const void* A, void* P, int64_t M, int64_t K, int64_t lda, int64_t ldp, sp24_dtype t, hipStream_t st);
sp24_status launch_mask_apply(const void* W, const void* meta, void* P, int64_t M, int64_t K, int64_t ldw, int64_t ldp, sp24_dtype t,
                              sp24_layout l, hipStream_t st);
sp24_status launch_permute_columns(const void* A, const void* perm, void* P, int64_t M, int64_t K, int64_t lda, int64_t ldp, sp24_dtype t,
                                   hipStream_t st);
sp24_status launch_permute_rows(const void* A, const void* perm, void* P, int64_t M, int64_t K, int64_t lda, int64_t ldp, sp24_dtype t,
                                hipStream_t st);
sp24_status launch_retained_magnitude(const void* A, const void* perm, double* out, int64_t M, int64_t K, int64_t lda, sp24_dtype t,
                                      hipStream_t st);
sp24_status launch_permute_search(const void* A, int32_t* perm, int64_t M, int64_t K, int64_t lda, sp24_dtype t, int sweeps, hipStream_t st);
// on a copy that lies column by column, in permute_search_workspace() bytes (0: not for this shape)
size_t permute_search_workspace(int64_t M, int64_t K, sp24_dtype t);
sp24_status launch_permute_search_columns(const void* A, int32_t* perm, int64_t M, int64_t K, int64_t lda, sp24_dtype t, int sweeps,
                                          void* workspace, hipStream_t st);
sp24_status launch_compress_masked(const void* W, const void* meta, void* V, int64_t M, int64_t K, int64_t ldw, sp24_dtype t,
                                   sp24_layout l, hipStream_t st);
sp24_status launch_decompress(const void* V, const void* meta, void* P, int64_t M, int64_t K, int64_t ldp, sp24_dtype t, sp24_layout l, hipStream_t st);

// Geometry of a convolution read as an implicit GEMM (Sec. 3.2: convolutions are GEMM-like operations; Sec. 4.2:
// inner dimension C x R x S): the second operand is never formed, element (k, n) of it is
//   X[img][oy*stride_h - pad_h + r][ox*stride_w - pad_w + s][c]   (zero outside the image)
// with k = (r*S + s)*C + c and n = (img*OH + oy)*OW + ox, X being NHWC.
struct ConvGeom {
    int on;                 // 0: plain matrix B
    int H, W, C, R, S, pad_h, pad_w, stride_h, stride_w, OH, OW;
};

// Problem description for the matrix-multiply kernels.  For the sparse product
// A = V and lda is unused; for the dense product meta is null.
struct MmArgs {
    const void* A;      // V (sparse) or dense A
    const void* meta;   // sparse only
    const void* B;
    void* D;
    int64_t M, N, K;
    int64_t lda, ldb, ldd; // elements
    sp24_dtype in, out;
    sp24_border bo;
    sp24_layout layout;    // sparse only
    bool sparse;
    ConvGeom conv;         // conv.on: B is the NHWC input X, N = n_img*OH*OW, K = R*S*C, bo / ldb unused
    Epilogue epi;          // epi.on: int8 inputs, scaled / re-quantised output (out = I8, F16, BF16 or F32)
    // K split across workgroups (tiled kernels only; k_slices > 1): slice s covers slice_steps whole 128-byte steps
    // from s * slice_steps on and writes its partial product, in the accumulator type, to image s of D
    // (M rows of ldd values each); out must then be F32 or I32, and conv and epi off.
    int k_slices, slice_steps;
    static constexpr bool kOwnStore = false;   // (arguments derived from these may bring their own way out)
    static constexpr bool kMMajorA = false;    // (dense: A as its transpose, a row of M for every k)
    static constexpr bool kPaddedColumns = false;      // (N-major B: its rows are whole 16-byte chunks whatever N is)
};

// General kernel: any M, N; both layouts; both B orders.  One wavefront per 32x32 tile of D.  Of the sparse products only
// those past the other kernels' index ranges come here.
sp24_status launch_mm_simple(const MmArgs& a, hipStream_t st);

// N-major B at any alignment, K split across the wavefronts of a workgroup; false in *handled for other problems.
sp24_status launch_mm_ksplit(const MmArgs& a, hipStream_t st, bool* handled);

// Sparse products and convolutions that the tiled kernels do not take, on tiles of their shape; false in *handled for
// other problems.
sp24_status launch_mm_staged(const MmArgs& a, hipStream_t st, bool* handled);

// Sparse 3x3 convolution of 8-bit inputs in chunks of 64 channels; false in *handled for other problems.
sp24_status launch_conv_narrow(const MmArgs& a, hipStream_t st, bool* handled);

// Sparse products with few columns or few tiles, K split across the wavefronts of a workgroup; false in *handled for
// operands it does not take.
sp24_status launch_mm_stream(const MmArgs& a, hipStream_t st, bool* handled);

// Columns of its tiles (of 32 rows) and workgroups it would launch
inline int stream_columns(const MmArgs& a) { return a.N <= 16 ? 16 : a.N <= 32 ? 32 : 64; }
inline int64_t stream_workgroups(const MmArgs& a) { return ((a.M + 31) / 32) * ((a.N + stream_columns(a) - 1) / stream_columns(a)); }

// Streaming kernel for N <= 32; returns false in *handled when the problem does not fit it.
sp24_status launch_mm_skinny(const MmArgs& a, hipStream_t st, bool* handled);

// Tiled kernels for large shapes; return false in *handled when the shape does not fit them.
sp24_status launch_mm_tiled(const MmArgs& a, hipStream_t st, bool* handled);

// D [M, N] (type out) = the sum, in slice order, of `slices` partial products (float or int32, M rows of ldw values
// each, images M * ldw values apart).
sp24_status launch_splitk_reduce(const void* partial, int slices, int64_t M, int64_t N, int64_t ldw, void* D, int64_t ldd, bool integer,
                                 sp24_dtype out, hipStream_t st);

// A launch has fewer than 2^32 threads along x (the runtime does not refuse more: it runs what the low 32 bits say).
inline int64_t most_groups(int threads) { return (((int64_t)1 << 32) - 1) / threads; }
// `groups` workgroups for each of `images`, one to a tile that a kernel finds from its number: SP24_ERR_SHAPE, and no launch, where it holds fewer
template <class F>
sp24_status launch_tiles(int64_t groups, int images, int threads, F&& launch)
{
    if (groups > most_groups(threads)) return SP24_ERR_SHAPE;
    launch(dim3((unsigned)groups, (unsigned)images), dim3((unsigned)threads));
    return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
}
// launch(first, grid) for as many launches as `groups` workgroups take, workgroup b of one being number first + b
template <class F>
sp24_status launch_in_parts(int64_t groups, int threads, F&& launch)
{
    if (groups == 0) return SP24_OK;
    const int64_t most = most_groups(threads);
    for (int64_t first = 0; first < groups; first += most) launch((unsigned)first, (unsigned)std::min(groups - first, most));
    return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
}

// ---- the operators around the products (N rows of H values unless said otherwise; ld* in elements) ----
struct RowsArgs {
    const void *X, *residual;
    const float* weight;                  // null: quantisation alone
    void *Y, *hidden;
    float *scale, *rstd;
    int64_t N, H, ldx, ldr, ldy, ldh;
    float eps;
    sp24_dtype t, out;
};
sp24_status launch_norm_rows(const RowsArgs& a, hipStream_t st);

struct NormGradArgs {
    const void *dY, *hidden, *dhidden;
    const float *weight, *rstd;
    void* dX;
    float *partial, *dweight;             // partial: norm_grad_groups() rows of H
    int64_t N, H, lddy, ldh, lddh, lddx;
    sp24_dtype t;
};
int64_t norm_grad_groups(int64_t N, int64_t H);
sp24_status launch_norm_grad(const NormGradArgs& a, hipStream_t st);

// out [segments][columns] = sums of rows of `partial` (rows x columns), all of them or (offsets) segment by segment, `unit` rows of the
// offsets to one of partial
sp24_status launch_column_sums(const float* partial, int64_t rows, int64_t columns, const int32_t* offsets, int segments, int unit, float* out,
                               hipStream_t st);

struct LinearGradArgs {
    const void *dY, *Z;                   // N rows of M values; Z as codes (zcode) with their scales
    const float* zscale;
    void *dZ, *dZt;
    float *partial, *dbias;               // partial: a row of M for every `unit` (16 or 64) rows
    const int32_t* offsets;
    int64_t M, N, lddy, ldz, lddz, lddzt;
    int act, experts, unit;
    sp24_dtype t, zcode;                  // zcode: t, or the 8-bit type
};
sp24_status launch_linear_grad(const LinearGradArgs& a, hipStream_t st);

constexpr int kSortAtOnce = 1 << 17;      // choices that one launch sorts (both sides measured in experts.hip); of more, parts of kSortPart
constexpr int kSortPart = 16384;
struct SortArgs {
    const int32_t* ids;                   // T choices
    int32_t *offsets, *slots, *rows, *workspace;      // workspace: experts words for every part where there are several
    int64_t T, R;
    int experts;
};
sp24_status launch_moe_sort(const SortArgs& a, hipStream_t st);

struct GatherArgs {
    const void* X;
    const float* scale;
    const int32_t* rows;
    void* Xs;
    float* scale_out;
    int64_t N, R, row_bytes, ldx_bytes, ldxs_bytes;
    int topk;
};
sp24_status launch_moe_gather(const GatherArgs& a, hipStream_t st);

struct CombineArgs {
    const void *Y, *residual;
    const int32_t* slots;
    const float* weights;                 // null: 1
    void* out;
    int64_t N, R, H, ldy, ldr, ldo;
    int topk;
    sp24_dtype t;
};
sp24_status launch_moe_combine(const CombineArgs& a, hipStream_t st);

struct CombineGradArgs {
    const void *dOut, *Y;
    const int32_t *rows, *slots;
    const float* weights;
    void* dY;
    float* dweights;
    int64_t N, R, H, lddo, ldy, lddy;
    int topk;
    sp24_dtype t;
};
sp24_status launch_moe_combine_grad(const CombineGradArgs& a, hipStream_t st);

struct RouteArgs {
    const void* logits;
    const float* bias;                    // null: 0
    int32_t* ids;
    float *weights, *scores;              // scores, load: null where not asked for
    int32_t* load;
    int64_t N, ldl;
    int experts, topk, groups, groups_kept, group_best, softmax, renormalise;
    float scale;
    sp24_dtype t;
};
sp24_status launch_moe_route(const RouteArgs& a, hipStream_t st);

struct RouteGradArgs {
    const void* logits;
    const int32_t* ids;
    const float *dweights, *dscores;      // dscores null: 0
    void* dlogits;
    int64_t N, ldl, lddl;
    int experts, topk, softmax, renormalise;
    float scale;
    sp24_dtype t;
};
sp24_status launch_moe_route_grad(const RouteGradArgs& a, hipStream_t st);

constexpr int kKeptBlock = SP24_CHECKPOINT_BLOCK;      // values of a row under one scale
__host__ __device__ inline int64_t kept_blocks(int64_t H) { return (H + kKeptBlock - 1) / kKeptBlock; }
struct KeepArgs {
    const void* X;
    void* codes;
    float* scale;                         // N x kept_blocks(H)
    int64_t N, H, ldx, ldc;
    sp24_dtype t, code;
};
sp24_status launch_checkpoint_rows(const KeepArgs& a, hipStream_t st);

struct RestoreArgs {
    const void* codes;
    const float* scale;
    const int32_t* rows;                  // null: row r of the codes
    void* out;
    int64_t N, R, H, ldc, ldo;            // N: rows of codes, R of out
    int topk, act;
    sp24_dtype code, t;
};
sp24_status launch_restore_rows(const RestoreArgs& a, hipStream_t st);

struct LinearArgs;                        // linear.hpp
struct GroupedArgs;
struct SegmentArgs;
sp24_status launch_linear(const LinearArgs& a, hipStream_t st);
sp24_status launch_linear_grouped(const GroupedArgs& a, hipStream_t st);
sp24_status launch_gemm_grouped(const SegmentArgs& a, int experts, hipStream_t st);
struct TokenArgs;
struct TokenSplit {
    int slices, steps;                    // of the tokens; steps of 64 tokens to one
    int64_t ldw;
    size_t bytes;                         // of the partial products (0: not split)
};
TokenSplit token_split(int64_t M, int64_t N, int64_t K);
// partial: token_split().bytes of a product that is to be split, or null
sp24_status launch_gemm_tokens(const TokenArgs& a, int experts, void* partial, hipStream_t st);
// the same of few tokens, the rows of B as `r` would restore them
sp24_status launch_gemm_codes(const TokenArgs& a, const RestoreArgs& r, int experts, hipStream_t st);

} // namespace sp24
