// The sparse product as a layer: rows per token out, bias, activation and residual in the epilogue, one scale per weight row and per token
// for 8-bit inputs; alone or for the segments of rows that belong to experts.
//   z[n][m] = (sum_k W[m][k] X[n][k]) * w_scale[m] * x_scale[n] + bias[m],  Y[n][m] = act(z[n][m]) + residual[n][m]
// The kernels are those of the plain product with another way out: in a matrix-core tile a lane holds runs of four rows m of one column n,
// which is a run of four values of a token's row.
#pragma once
#include <algorithm>

#include "mm_operands.hpp"
#include "rowops.hpp"

namespace sp24 {

struct LinearArgs : MmArgs {            // MmArgs::B = X, D = Y, ldd = ldy; epi.w_scale and epi.bias, epi.on unused
    static constexpr bool kOwnStore = true;
    const float* x_scale;               // N values, or null
    const void* residual;               // N x M of the output type, or null
    void* Z;                            // receives z in the output type, or null
    int64_t ldr, ldz;
    int act;

    template <int BM, int BN> __device__ __forceinline__ bool enter(int, int&) { return true; }
    template <int DT, int COUNT> struct way_out;
    // Bias and scales of a tile's BM features wait in LDS for the way out: transferred ahead of everything else, there with the first operands.
    template <int DT, int BM> static constexpr int vector_bytes() { return (is8<DT> ? 2 : 1) * BM * 4; }
    template <int DT, int BM, int NW> __device__ __forceinline__ void fetch_vectors(uint8_t* lds, int64_t m0, int wave, int lane) const
    {
#pragma unroll
        for (int v = 0; v < (is8<DT> ? 2 : 1); ++v) {
            const float* const p = v == 0 ? epi.bias : epi.w_scale;
#pragma unroll
            for (int x = 0; x < (BM / 64 + NW - 1) / NW; ++x) {
                const int part = wave + x * NW;
                if (!p || part >= BM / 64) continue;
                lds_dma4_addr(reinterpret_cast<const uint8_t*>(p + min(m0 + part * 64 + lane, M - 1)), lds + v * BM * 4 + part * 256);
            }
        }
    }
    template <int TM> static constexpr int wave_bytes();
    // vectors: where fetch_vectors put them, the wavefront's first feature of BM being `first`
    template <int DT, int TM, int TN>
    __device__ __forceinline__ void store_wave(typename acc_of<DT>::type (&acc)[TM][TN], uint8_t* scratch, const uint8_t* vectors, int BM, int first,
                                               int64_t row_base, int64_t col_base, int lane) const;
};

constexpr int kSegmentRows = 16;        // segments begin at multiples of this

// rows first .. last - 1 of segment e, whole sixteens inside the `rows` there are
__device__ __forceinline__ void segment_of(const int32_t* offsets, int e, int64_t rows, int64_t& first, int64_t& last)
{
    first = min(max((int64_t)offsets[e], (int64_t)0), rows) / kSegmentRows * kSegmentRows;
    last = min(max((int64_t)offsets[e + 1], first), rows) / kSegmentRows * kSegmentRows;
}

// Tiles of `width` rows that a launch has to provide for, whatever the segments are: every segment may end inside a tile, and one more set
// covers the rows behind the last.
inline int64_t grouped_tiles(int64_t rows, int experts, int width)
{
    const int64_t live = std::min<int64_t>(experts, rows / kSegmentRows);
    return (rows + live * (width - kSegmentRows)) / width + 1;
}

// The same for experts: rows offsets[e] .. offsets[e + 1] - 1 of X and Y belong to expert e, whose M rows of weights follow those of the
// experts before it.  N counts all rows; those of no segment are written zero.
struct GroupedArgs : LinearArgs {
    const int32_t* offsets;
    int experts;

    // The tile's place among the segments: the operands become those of its expert, N the rows of its segment, tn the tile in it.
    // false: not a tile of the product (rows behind the last segment are written here).
    template <int BM, int BN> __device__ __forceinline__ bool enter(int tm, int& tn)
    {
        const int lane = threadIdx.x & 63;
        int before = 0;
        int64_t end = 0;
        for (int e0 = 0; e0 < experts; e0 += 64) {
            const int e = e0 + lane;
            int64_t first = 0, last = 0;
            if (e < experts) segment_of(offsets, e, N, first, last);
            const int tiles = (int)((last - first + BN - 1) / BN);
            int upto = tiles;                                     // tiles of this and the earlier lanes
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int t = __shfl_up(upto, d);
                if (lane >= d) upto += t;
            }
            const uint64_t hit = __ballot(tn < before + upto);
            if (hit != 0) {
                const int l = __builtin_ctzll(hit), expert = e0 + l;
                tn = __builtin_amdgcn_readfirstlane(tn - before - __shfl(upto - tiles, l));
                const int64_t from = __builtin_amdgcn_readfirstlane((int)__shfl((int)first, l)), to = __builtin_amdgcn_readfirstlane((int)__shfl((int)last, l));
                const int es = esize_of(in), os = esize_of(out);
                A = reinterpret_cast<const uint8_t*>(A) + expert * (M * (K / 2) * es);
                meta = reinterpret_cast<const uint8_t*>(meta) + expert * (M * (K / 8));
                B = reinterpret_cast<const uint8_t*>(B) + from * ldb * es;
                D = reinterpret_cast<uint8_t*>(D) + from * ldd * os;
                if (Z) Z = reinterpret_cast<uint8_t*>(Z) + from * ldz * os;
                if (epi.w_scale) epi.w_scale += expert * M;
                if (epi.bias) epi.bias += expert * M;
                if (x_scale) x_scale += from;
                N = to - from;
                return true;
            }
            before += __shfl(upto, 63);
            int reach = (int)last;                                // (segments lie one behind the other: the furthest end)
#pragma unroll
            for (int d = 32; d > 0; d /= 2) reach = max(reach, __shfl_xor(reach, d));
            end = max(end, (int64_t)reach);
        }
        zero_rows<BM, BN>(end + (int64_t)(tn - before) * BN, (int64_t)tm * BM);
        return false;
    }
    // rows first .. first + BN - 1 (as far as there are) of Y and Z, columns m0 .. m0 + BM - 1: zeros
    template <int BM, int BN> __device__ __forceinline__ void zero_rows(int64_t first, int64_t m0) const
    {
        const int64_t columns = min((int64_t)BM, M - m0);
        for (int i = threadIdx.x; i < BN * (BM / 8); i += blockDim.x) {
            const int64_t row = first + i / (BM / 8), c = (int64_t)(i % (BM / 8)) * 8;
            if (row >= N || c >= columns) continue;
            const int n = (int)min(columns - c, (int64_t)8);
            const float none[8] = {};
            auto put8 = [&](void* p, int64_t ld) {
                if (out == SP24_F32) store_values8<SP24_F32>(p, row * ld + m0 + c, n, none);
                else store_values8<SP24_BF16>(p, row * ld + m0 + c, n, none);      // (zeros of either 16-bit type)
            };
            put8(D, ldd);
            if (Z) put8(Z, ldz);
        }
    }
};

// The dense product of every segment: K (the rows) runs over segment blockIdx.y, whose result is that image of D.
struct SegmentArgs : MmArgs {
    const int32_t* offsets;

    template <int BM, int BN> __device__ __forceinline__ bool enter(int, int&)
    {
        const int es = esize_of(in), e = blockIdx.y;
        int64_t first, last;
        segment_of(offsets, e, K, first, last);
        A = reinterpret_cast<const uint8_t*>(A) + first * es;
        B = reinterpret_cast<const uint8_t*>(B) + first * ldb * es;
        D = reinterpret_cast<uint8_t*>(D) + e * M * ldd * esize_of(out);
        K = last - first;
        return true;
    }
};

// N neighbouring values of one row of the output, in registers: the first `n` of them.
template <int COUNT>
__device__ __forceinline__ void load_row_values(const void* p, int64_t at, int n, sp24_dtype t, float (&v)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = 0.0f;
    if constexpr (COUNT == 8) {
        if (t == SP24_F32) values_of(load_raw8<SP24_F32>(p, at, n), v);
        else {
            const raw8<SP24_BF16> r = load_raw8<SP24_BF16>(p, at, n);
            if (t == SP24_BF16) values_of<SP24_BF16>(r, v);
            else values_of<SP24_F16>(raw8<SP24_F16>{{r.q[0]}}, v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (i < n) v[i] = t == SP24_F32 ? load_value<SP24_F32>(p, at + i) : t == SP24_BF16 ? load_value<SP24_BF16>(p, at + i) : load_value<SP24_F16>(p, at + i);
    }
}

// past_l2: the values lie on 16-byte boundaries and are not read again by this launch
template <int COUNT>
__device__ __forceinline__ void store_row_values(void* p, int64_t at, int n, sp24_dtype t, bool past_l2, const float (&v)[COUNT])
{
    if constexpr (COUNT == 8) {
        if (past_l2 && n >= 8 && t != SP24_F32) {
            uint4v q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = t == SP24_BF16 ? pack_out16<SP24_BF16>(v[2 * i], v[2 * i + 1]) : pack_out16<SP24_F16>(v[2 * i], v[2 * i + 1]);
            __builtin_nontemporal_store(q, reinterpret_cast<uint4v*>(reinterpret_cast<uint16_t*>(p) + at));
            return;
        }
        if (t == SP24_F32) store_values8<SP24_F32>(p, at, n, v);
        else if (t == SP24_BF16) store_values8<SP24_BF16>(p, at, n, v);
        else store_values8<SP24_F16>(p, at, n, v);
    } else {
        if (t == SP24_F32) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                if (i < n) reinterpret_cast<float*>(p)[at + i] = v[i];
            return;
        }
        uint32_t q[COUNT / 2];
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i) q[i] = t == SP24_BF16 ? pack_out16<SP24_BF16>(v[2 * i], v[2 * i + 1]) : pack_out16<SP24_F16>(v[2 * i], v[2 * i + 1]);
        uint16_t* const to = reinterpret_cast<uint16_t*>(p) + at;
        if (n >= COUNT) {
            typedef uint32_t words __attribute__((ext_vector_type(COUNT / 2)));
            words w;
            if constexpr (COUNT == 2) w = q[0];
            else {
#pragma unroll
                for (int i = 0; i < COUNT / 2; ++i) w[i] = q[i];
            }
            store_to(to, w);
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                if (i < n) to[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
        }
    }
}

// The way out of COUNT neighbouring values of token n's row, from feature m on (`have` of them exist): `v` are the sums.
template <int DT, int COUNT>
__device__ __forceinline__ void finish_row_values(const LinearArgs& a, int64_t n, int64_t m, int have, const float (&scale)[COUNT], const float (&bias)[COUNT],
                                                  float x_scale, const float (&more)[COUNT], bool past_l2, float (&v)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        if constexpr (is8<DT>) v[i] = __builtin_fmaf(v[i] * scale[i], x_scale, bias[i]);
        else v[i] += bias[i];
    }
    if (a.Z) store_row_values(a.Z, n * a.ldz + m, have, a.out, past_l2, v);
    activate(v, a.act);
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] += more[i];
    }
    store_row_values(a.D, n * a.ldd + m, have, a.out, past_l2, v);
}

// COUNT values of a vector over the features, `otherwise` where there is none
template <int COUNT>
__device__ __forceinline__ void load_feature_values(const float* p, int64_t m, int have, float otherwise, float (&v)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = p && i < have ? p[m + i] : otherwise;
}

// COUNT neighbouring features of token n's row on their way out; what has to be read for them can be asked for before the sums are there.
template <int DT, int COUNT>
struct LinearArgs::way_out {
    float scale[COUNT], bias[COUNT], more[COUNT], x_scale;
    __device__ __forceinline__ void fetch(const LinearArgs& a, int64_t n, int64_t m)
    {
        const int have = (int)min(a.M - m, (int64_t)COUNT);
        load_feature_values(is8<DT> ? a.epi.w_scale : nullptr, m, have, 1.0f, scale);
        load_feature_values(a.epi.bias, m, have, 0.0f, bias);
        x_scale = is8<DT> && a.x_scale ? a.x_scale[n] : 1.0f;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) more[i] = 0.0f;
        if (a.residual) load_row_values(a.residual, n * a.ldr + m, have, a.out, more);
    }
    __device__ __forceinline__ void finish(const LinearArgs& a, int64_t n, int64_t m, float (&v)[COUNT]) const
    {
        finish_row_values<DT>(a, n, m, (int)min(a.M - m, (int64_t)COUNT), scale, bias, x_scale, more, false, v);
    }
};

// f(integral_constant<int, 0>{}), ..., f(integral_constant<int, N - 1>{})
template <int N, class F>
__device__ __forceinline__ void count_up(F&& f)
{
    if constexpr (N > 0) {
        count_up<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// A wavefront's tile on its way out, 32 tokens at a time: the sums go to LDS in binary32 as rows of 32 TM features and come back eight
// neighbouring ones to a lane, so that every global access is 16 bytes and covers whole lines of a token's row.  Rows are 16 bytes
// longer than their values: 16 lanes that write 16 bytes of 16 rows, or read 16 of 2 rows, meet every bank once.  4096 x 8192 x 1024
// bf16 with bias: 46.7 us without an activation, 54 to 56 with GELU.
template <int TM> constexpr int LinearArgs::wave_bytes() { return 32 * (TM * 128 + 16); }

template <int DT, int TM, int TN>
__device__ __forceinline__ void LinearArgs::store_wave(typename acc_of<DT>::type (&acc)[TM][TN], uint8_t* scratch, const uint8_t* vectors, int BM, int first,
                                                       int64_t row_base, int64_t col_base, int lane) const
{
    constexpr int kPitch = TM * 128 + 16, CH = 4 * TM;            // chunks of eight features to a row
    constexpr int IT = 32 * CH / 64, kRows = 64 / CH;             // instructions to 32 tokens, tokens to one
    const int r = lane & 31, q = lane >> 5, c = lane % CH;
    const int64_t m = row_base + c * 8;
    const int have = (int)min(M - m, (int64_t)8);
    // Y (and Z) go past the L2, which keeps the panels that neighbouring tiles share: 4096 x 8192 x 1024 bf16 with GELU 54.7 -> 52.8 us,
    // 8192 x 4096 x 4096 with SiLU 143.6 -> 132.1
    const bool past_l2 = ((reinterpret_cast<uintptr_t>(D) | reinterpret_cast<uintptr_t>(Z)) & 15u) == 0 && ldd % 8 == 0 && (!Z || ldz % 8 == 0);
    float scale[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float* const v = reinterpret_cast<const float*>(vectors) + first + c * 8 + i;
        b[i] = epi.bias ? v[0] : 0.0f;
        scale[i] = is8<DT> && epi.w_scale ? v[BM] : 1.0f;
    }
    // (as calls, not a loop: a loop of this size the compiler may leave rolled, and then keeps the sums in memory)
    count_up<TN>([&](auto j_c) __attribute__((always_inline)) {
        constexpr int j = decltype(j_c)::value;
        const int64_t n0 = col_base + j * 32 + lane / CH;
        float more[IT][8], xs[IT];
#pragma unroll
        for (int it = 0; it < IT; ++it) {                          // on their way while the sums take the turn through LDS
            const int64_t n = min(n0 + it * kRows, N - 1);
            xs[it] = is8<DT> && x_scale ? x_scale[n] : 1.0f;
            if (residual) load_row_values(residual, n * ldr + m, have, out, more[it]);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4v v = {(float)acc[i][j][4 * g], (float)acc[i][j][4 * g + 1], (float)acc[i][j][4 * g + 2], (float)acc[i][j][4 * g + 3]};
                *reinterpret_cast<float4v*>(scratch + r * kPitch + (i * 32 + 8 * g + 4 * q) * 4) = v;
            }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int64_t n = n0 + it * kRows;
            const float4v lo = *reinterpret_cast<const float4v*>(scratch + (it * kRows + lane / CH) * kPitch + c * 32);
            const float4v hi = *reinterpret_cast<const float4v*>(scratch + (it * kRows + lane / CH) * kPitch + c * 32 + 16);
            if (n >= N || have <= 0) continue;
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            finish_row_values<DT>(*this, n, m, have, scale, b, xs[it], more[it], past_l2, v);
        }
    });
}

// ---- host side: the tiled, the staged and the streaming kernels, compiled per input type ----
// (t128x128_one: six stages, one workgroup to a unit; t128x128: three stages, two)
enum class LayerTile { stream, t64x32, t128x64, t128x128, t128x128_one, t256x128, t256x256 };
template <int DT, class ARGS> sp24_status layer_tiled(const ARGS& a, LayerTile tile, hipStream_t st);
template <int DT, class ARGS> sp24_status layer_staged(const ARGS& a, hipStream_t st);
sp24_status launch_linear_stream(const LinearArgs& a, hipStream_t st);
sp24_status launch_grouped_stream(const GroupedArgs& a, hipStream_t st);

// f(integral_constant<int, the input type>{})
template <class F>
sp24_status by_input(const MmArgs& a, F&& f)
{
    if (a.in == SP24_I8) return f(std::integral_constant<int, SP24_I8>{});
    if (a.in == SP24_F8) return f(std::integral_constant<int, SP24_F8>{});
    if (a.in == SP24_F16) return f(std::integral_constant<int, SP24_F16>{});
    return f(std::integral_constant<int, SP24_BF16>{});
}

} // namespace sp24
