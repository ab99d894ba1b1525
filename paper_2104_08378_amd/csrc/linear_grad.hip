// What follows from the gradient of a layer's result: dZ = dY act'(Z) as rows per token, the same transposed (the first operand of the
// weights' gradient), and the bias's gradient, the sum of dZ over the rows of a segment.
//
// Bound by memory: dY and Z are read once, both forms of dZ written once.  A workgroup takes 64 rows x 64 (128) values through LDS in binary32,
// so that the sums see them unrounded; rows of 65 (129) words there, of which the columns' reads (8 rows x 8 a wavefront) find no
// bank twice, and the rows' writes none (two).  Sums: 16 rows (the unit of segments) in row order, then those in order.
// 4096 x 4096 bf16 with GELU, the sums' second kernel included: 31.6 us, 134 MB at 4.2 TB/s; without an activation 14.9, 67 MB at 4.5.  Z kept in 8 bits and
// no transposed form, 8192 x 4096: 32 us, 161 MB at 5.0.
//
// dZ is rounded to 16 bits, which both of its products read (the matrix instructions' operands): gradients of 4096 x 1024 weights from 4096
// tokens are off by 0.0023 of their size in bf16, where rounding the results alone leaves 0.0017.  The bias's gradient sums unrounded values.
#include "kept.hpp"
#include "launch.hpp"
#include "linear.hpp"

namespace sp24 {

constexpr int kGradTile = 64;           // rows of a tile
constexpr int kFewExperts = 32;         // whose segments four groups of threads go through one after the other

// ZT: what Z is held in, the values' type or codes with a scale for each block of 128.  FEW: there is one tile of rows, and the sums need no
// second launch: they are added sixteen rows at a time, in row order.
template <int T, int ZT, int WIDTH, int ROWS, bool FEW>
__global__ __launch_bounds__(ROWS * WIDTH / 16) void k_linear_grad(LinearGradArgs a, int tiles_m, unsigned from)
{
    constexpr int kPitch = WIDTH + 1, CH = WIDTH / 8;
    constexpr int kAtOnce = ROWS / 2;                                  // rows that the threads load together
    __shared__ float tile[ROWS * kPitch];
    __shared__ float part[ROWS / 16][WIDTH];
    const int tid = threadIdx.x;
    const unsigned at = from + blockIdx.x;
    const int64_t m0 = (int64_t)(at % tiles_m) * WIDTH, n0 = (int64_t)(at / tiles_m) * ROWS;
    const int c = tid % CH;
    const int64_t m = m0 + c * 8;
    const int have = (int)min(a.M - m, (int64_t)8);
    raw8<T> dy[2] = {}, z[2] = {};
    uint2v codes[2] = {};
    float scale[2] = {};
#pragma unroll
    for (int it = 0; it < 2; ++it) {
        const int64_t n = n0 + it * kAtOnce + tid / CH;
        if (n < a.N && have > 0) {
            dy[it] = load_raw8<T>(a.dY, n * a.lddy + m, have);
            if (a.act != SP24_ACT_NONE) {
                if constexpr (is8<ZT>) {
                    codes[it] = load_codes8<false>(reinterpret_cast<const uint8_t*>(a.Z) + n * a.ldz + m, have);
                    scale[it] = a.zscale[n * kept_blocks(a.M) + m / kKeptBlock];
                } else z[it] = load_raw8<T>(a.Z, n * a.ldz + m, have);
            }
        }
    }
#pragma unroll
    for (int it = 0; it < 2; ++it) {
        const int t = it * kAtOnce + tid / CH;
        float v[8], x[8];
        values_of<T>(dy[it], v);
        if (a.act != SP24_ACT_NONE) {
            if constexpr (is8<ZT>) kept_values8<ZT>(codes[it], scale[it], x);
            else values_of<T>(z[it], x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= activation_slope(x[i], a.act);
        }
        if (a.dZ && n0 + t < a.N && have > 0) store_values8<T>(a.dZ, (n0 + t) * a.lddz + m, have, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[t * kPitch + c * 8 + i] = v[i];
    }
    __syncthreads();
    if (a.dZt) {
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const int f = it * (WIDTH / 2) + tid / (ROWS / 8), t = tid % (ROWS / 8) * 8;
            const int rows = (int)min(a.N - n0 - t, (int64_t)8);
            if (m0 + f >= a.M || rows <= 0) continue;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[(t + i) * kPitch + f];
            store_values8<T>(a.dZt, (m0 + f) * a.lddzt + n0 + t, rows, v);
        }
    }
    if constexpr (FEW) {
        const int f = tid % WIDTH, p = tid / WIDTH;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += tile[(p * 16 + i) * kPitch + f];           // (rows past N are zeros)
        part[p][f] = sum;
        __syncthreads();
        if (m0 + f >= a.M) return;
        if (!a.offsets) {
            float total = 0.0f;
            for (int k = 0; p == 0 && k < ROWS / 16; ++k) total += part[k][f];
            if (p == 0) a.dbias[m0 + f] = total;
        } else {
            for (int e = p; e < a.experts; e += ROWS / 16) {
                int64_t from_row, to_row;
                segment_of(a.offsets, e, a.N, from_row, to_row);
                float total = 0.0f;
                for (int64_t k = from_row / 16; k < to_row / 16; ++k) total += part[k][f];
                a.dbias[(int64_t)e * a.M + m0 + f] = total;
            }
        }
    } else if (a.partial) {
        const int f = tid % WIDTH, p = tid / WIDTH;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += tile[(p * 16 + i) * kPitch + f];       // (rows past N are zeros)
        if (a.unit == 16) {
            const int64_t row = n0 / 16 + p;
            if (m0 + f < a.M && row * 16 < a.N) a.partial[row * a.M + m0 + f] = sum;
        } else {
            part[p][f] = sum;
            __syncthreads();
            if (p == 0 && m0 + f < a.M) a.partial[n0 / ROWS * a.M + m0 + f] = ((part[0][f] + part[1][f]) + part[2][f]) + part[3][f];
        }
    }
}

template <int WIDTH, int ROWS, bool FEW>
static sp24_status run_linear_grad(const LinearGradArgs& a, hipStream_t st)
{
    const int64_t tiles_m = (a.M + WIDTH - 1) / WIDTH, tiles_n = (a.N + ROWS - 1) / ROWS;
    constexpr int kThreads = ROWS * WIDTH / 16;
    return launch_in_parts(tiles_m * tiles_n, kThreads, [&](unsigned from, unsigned grid) {
        auto run = [&](auto t) {
            constexpr int T = decltype(t)::value;
            if (a.zcode == SP24_I8) k_linear_grad<T, SP24_I8, WIDTH, ROWS, FEW><<<grid, kThreads, 0, st>>>(a, (int)tiles_m, from);
            else if (a.zcode == SP24_F8) k_linear_grad<T, SP24_F8, WIDTH, ROWS, FEW><<<grid, kThreads, 0, st>>>(a, (int)tiles_m, from);
            else if constexpr (!FEW) k_linear_grad<T, T, WIDTH, ROWS, FEW><<<grid, kThreads, 0, st>>>(a, (int)tiles_m, from);
        };
        if (a.t == SP24_F16) run(std::integral_constant<int, SP24_F16>{});
        else run(std::integral_constant<int, SP24_BF16>{});
    });
}

sp24_status launch_linear_grad(const LinearGradArgs& a, hipStream_t st)
{
    // One tile of 64, 128 or 256 rows, Z kept in 8 bits (the sums beside a 16-bit Z keep their order, and with it their bits): 64 x 2048 5.9 -> 4.1 us, 128 x 2048
    // 6.1 -> 4.2, 256 x 2048 6.2 -> 5.3, of segments 6.4 -> 4.4, 6.5 -> 4.5 and 6.6 -> 5.7.  (Tiles of 64 one after the other in a workgroup: 128 rows 7.1, 256 rows 12.4.)
    if (a.zcode != a.t && a.dbias && a.N > 0 && a.N <= 256 && a.experts <= kFewExperts) {
        if (a.N <= 64) return run_linear_grad<64, 64, true>(a, st);
        return a.N <= 128 ? run_linear_grad<64, 128, true>(a, st) : run_linear_grad<64, 256, true>(a, st);
    }
    // Large ones with an activation, whose two operands come in rows of 256 bytes a tile then: 4096 x 4096 with GELU 35.6 -> 32.9 us.  Without
    // one 15.2 and 16.0, and few tiles (4096 x 512) 8.7 and 9.0.
    const bool wide = a.act != SP24_ACT_NONE && a.M * a.N >= (int64_t)1 << 22;
    const sp24_status s = wide ? run_linear_grad<128, kGradTile, false>(a, st) : run_linear_grad<64, kGradTile, false>(a, st);
    if (s != SP24_OK || !a.dbias || a.M == 0) return s;
    return launch_column_sums(a.partial, (a.N + a.unit - 1) / a.unit, a.M, a.offsets, a.offsets ? a.experts : 1, a.unit, a.dbias, st);
}

} // namespace sp24
