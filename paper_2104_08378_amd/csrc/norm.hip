// Root-mean-square norm of rows (with the residual added in front and 8-bit rows with a scale each behind), the quantisation of rows
// alone, and the norm's gradients.
//
//   h = x + r,  y = h rstd w,  rstd = (mean h^2 + eps)^-1/2;   8-bit: scale = max|y| / top, code = y (top / max|y|) rounded
//   g = w dy,  dx = rstd (g - h rstd^2 mean(g h)) + dh,  dw = sum over the rows of dy h rstd
//
// Bound by memory: a row is read once, stays in registers (eight values a lane and chunk, in binary32 as all sums are) and is written
// once.  A workgroup takes a row after the other and keeps its weights.  8192 x 4096 bf16 with residual to 8-bit floats: 49 us, 235 MB at 4.8 TB/s
// (a large copy reaches 5.4); to bf16 54 (5.0); 4000 rows of 4095, at odd addresses, 44 (3.0); 16 rows of 8192 3.5 us, little but the launch.
// The quantisation alone: 8192 x 4096 bf16 21 us, 101 MB at 4.8 TB/s; 16 x 8192 3.2.
// Gradients with the column sums: 4096 x 1024 11.8 us, 16000 x 1024 31 (4.3 TB/s).
//
// `hidden`, the residual stream, and the rows y are rounded once, to the caller's type, in which the next call reads them; the norm
// itself goes on with the unrounded h.
#include <algorithm>

#include "launch.hpp"
#include "rowops.hpp"

namespace sp24 {

// the value that 8-bit codes reach at the largest magnitude of their row
template <int OUT> constexpr float top_code() { return OUT == SP24_I8 ? 127.0f : 448.0f; }
constexpr float kLeastMagnitude = 7.888609052210118e-31f;       // 2^-100: a row below it has its codes taken against it

template <int OUT, bool WHOLE>
__device__ __forceinline__ void store_codes8(void* p, int64_t first, int n, const float (&v)[8])
{
    uint8_t* at = reinterpret_cast<uint8_t*>(p) + first;
    uint2v q = {0u, 0u};
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        if constexpr (OUT == SP24_I8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[d] |= ((uint32_t)(int)__builtin_rintf(v[4 * d + i]) & 0xFFu) << (8 * i);
        } else {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * d], v[4 * d + 1], 0, false);
            q[d] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * d + 2], v[4 * d + 3], w, true);
        }
    }
    if (WHOLE || n >= 8) store_to(at, q);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) at[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
    }
}

// C: chunks of eight values a thread holds; thread t those at (c * blockDim.x + t) * 8.  WHOLE: rows of whole chunks (the code for a
// part of one at every load and store costs registers that the many rows in flight need).  MOST: threads at most
template <int T, int OUT, int C, bool NORM, bool WHOLE, int MOST>
__global__ __launch_bounds__(MOST) void k_norm_rows(RowsArgs a)
{
    constexpr bool KEEP = C <= 2;                                // the weights of all rows in registers; else from the L2, row by row
    __shared__ uint32_t cells[3][16];
    const int H = (int)a.H;
    float w[KEEP ? C : 1][8];
    int n[C];                                                    // values of the chunk that exist
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int first = (c * blockDim.x + threadIdx.x) * 8;
        n[c] = WHOLE ? (first < H ? 8 : 0) : min(H - first, 8);
        if (NORM && KEEP && n[c] > 0) load_floats8<WHOLE>(a.weight, first, n[c], w[c]);
    }
    int parity = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        raw8<T> x[C], r[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int first = (c * blockDim.x + threadIdx.x) * 8;
            if (n[c] > 0) x[c] = load_raw8<T, WHOLE>(a.X, row * a.ldx + first, n[c]);
            if (NORM && a.residual && n[c] > 0) r[c] = load_raw8<T, WHOLE>(a.residual, row * a.ldr + first, n[c]);
        }
        float h[C][8], sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (n[c] <= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = 0.0f;
                continue;
            }
            values_of<T>(x[c], h[c]);
            if constexpr (NORM) {
                if (a.residual) {
                    float more[8];
                    values_of<T>(r[c], more);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[c][i] += more[i];
                }
                // (rounded to the rows' type here; the norm goes on with the unrounded sum)
                if (a.hidden) store_values8<T, WHOLE>(a.hidden, row * a.ldh + (c * blockDim.x + threadIdx.x) * 8, n[c], h[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[c][i], h[c][i], sum);
            }
        }
        float rstd = 1.0f, power = 1.0f, rest = 1.0f;            // rstd = power * rest, a power of two and a factor of 1 to 2
        if constexpr (NORM) {
            const float square = __uint_as_float(over_workgroup<add_f>(__float_as_uint(sum), cells[parity]));
            parity ^= 1;
            rstd = 1.0f / __builtin_sqrtf(square / (float)H + a.eps);
            if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
            if constexpr (is8<OUT>) {
                power = __uint_as_float(__float_as_uint(rstd) & 0x7F800000u);
                rest = __uint_as_float((__float_as_uint(rstd) & 0x007FFFFFu) | 0x3F800000u);
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (n[c] > 0) {
                    if (!KEEP) load_floats8<WHOLE>(a.weight, (c * blockDim.x + threadIdx.x) * 8, n[c], w[0]);
                    const float common = is8<OUT> ? power : rstd;
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * common * w[KEEP ? c : 0][i];
                }
        }
        if constexpr (is8<OUT>) {
            // Codes are a row's values over their largest, in which rstd cancels: two roundings less on the way to each.  Its power of two
            // rounds nothing and stays, so that h w passes no end of binary32 that y itself keeps within.
            // Magnitudes go by their bit patterns, in which a NaN is the largest: it reaches the scale, and no row hides one.
            // (Values past the row's end are zeros.)
            uint32_t most = 0;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = max(most, (WHOLE ? n[c] > 0 : i < n[c]) ? __float_as_uint(h[c][i]) & 0x7FFFFFFFu : 0u);
            const float largest = __uint_as_float(over_workgroup<max_u>(most, cells[2])), top = largest * rest;
            if (!NORM) __syncthreads();                          // (the norm's sum has a barrier between two uses of the cells)
            if (threadIdx.x == 0) a.scale[row] = (top < kLeastMagnitude ? kLeastMagnitude : top) / top_code<OUT>();
            const float inv = top < kLeastMagnitude ? rest * (top_code<OUT>() / kLeastMagnitude) : top_code<OUT>() / largest;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (n[c] <= 0) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] *= inv;
                store_codes8<OUT, WHOLE>(a.Y, row * a.ldy + (c * blockDim.x + threadIdx.x) * 8, n[c], h[c]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (n[c] > 0) store_values8<OUT, WHOLE>(a.Y, row * a.ldy + (c * blockDim.x + threadIdx.x) * 8, n[c], h[c]);
        }
    }
}

// The gradients.  A workgroup's share of dw stays in registers over its rows and goes to its row of `partial`.
template <int T, int C, bool WHOLE, int MOST>
__global__ __launch_bounds__(MOST) void k_norm_grad(NormGradArgs a)
{
    constexpr bool KEEP = C <= 2;
    __shared__ uint32_t cells[2][16];
    const int H = (int)a.H;
    float w[KEEP ? C : 1][8], dw[C][8];
    int n[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int first = (c * blockDim.x + threadIdx.x) * 8;
        n[c] = WHOLE ? (first < H ? 8 : 0) : min(H - first, 8);
        if (KEEP && n[c] > 0) load_floats8<WHOLE>(a.weight, first, n[c], w[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.0f;
    }
    int parity = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        raw8<T> dy_raw[C], h_raw[C], dh_raw[C];
        const float rstd = a.rstd[row];
        float along = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int first = (c * blockDim.x + threadIdx.x) * 8;
            if (n[c] <= 0) continue;
            dy_raw[c] = load_raw8<T, WHOLE>(a.dY, row * a.lddy + first, n[c]);
            h_raw[c] = load_raw8<T, WHOLE>(a.hidden, row * a.ldh + first, n[c]);
            if (a.dhidden) dh_raw[c] = load_raw8<T, WHOLE>(a.dhidden, row * a.lddh + first, n[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (n[c] <= 0) continue;
            float dy[8], h[8];
            values_of<T>(dy_raw[c], dy);
            values_of<T>(h_raw[c], h);
            if (!KEEP) load_floats8<WHOLE>(a.weight, (c * blockDim.x + threadIdx.x) * 8, n[c], w[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = dy[i] * h[i];
                if (WHOLE || i < n[c]) along = __builtin_fmaf(t, w[KEEP ? c : 0][i], along);
                dw[c][i] = __builtin_fmaf(t, rstd, dw[c][i]);
            }
        }
        along = __uint_as_float(over_workgroup<add_f>(__float_as_uint(along), cells[parity]));
        parity ^= 1;
        const float k = rstd * rstd * (along / (float)H);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (n[c] <= 0) continue;
            float dy[8], h[8], dx[8];
            values_of<T>(dy_raw[c], dy);
            values_of<T>(h_raw[c], h);
            if (!KEEP) load_floats8<WHOLE>(a.weight, (c * blockDim.x + threadIdx.x) * 8, n[c], w[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) dx[i] = rstd * (dy[i] * w[KEEP ? c : 0][i] - h[i] * k);
            if (a.dhidden) {
                float dh[8];
                values_of<T>(dh_raw[c], dh);
#pragma unroll
                for (int i = 0; i < 8; ++i) dx[i] += dh[i];
            }
            store_values8<T, WHOLE>(a.dX, row * a.lddx + (c * blockDim.x + threadIdx.x) * 8, n[c], dx);
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (n[c] > 0) store_values8<SP24_F32, WHOLE>(a.partial, (int64_t)blockIdx.x * a.H + (c * blockDim.x + threadIdx.x) * 8, n[c], dw[c]);
}

// The same with a wavefront to a row: no barriers on the way, and the shares of the eight wavefronts are added at the end.
constexpr int kGradWaves = 8;
template <int T, int C>
__global__ __launch_bounds__(64 * kGradWaves) void k_norm_grad_short(NormGradArgs a)
{
    __shared__ float share[kGradWaves / 2][C * 512];
    const int H = (int)a.H, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float dw[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.x * kGradWaves + wave; row < a.N; row += (int64_t)gridDim.x * kGradWaves) {
        raw8<T> dy_raw[C], h_raw[C], dh_raw[C];
        float w[C][8];
        const float rstd = a.rstd[row];
        float along = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int first = (c * 64 + lane) * 8;
            if (first >= H) continue;
            dy_raw[c] = load_raw8<T, true>(a.dY, row * a.lddy + first, 8);
            h_raw[c] = load_raw8<T, true>(a.hidden, row * a.ldh + first, 8);
            if (a.dhidden) dh_raw[c] = load_raw8<T, true>(a.dhidden, row * a.lddh + first, 8);
            load_floats8<true>(a.weight, first, 8, w[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if ((c * 64 + lane) * 8 >= H) continue;
            float dy[8], h[8];
            values_of<T>(dy_raw[c], dy);
            values_of<T>(h_raw[c], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = dy[i] * h[i];
                along = __builtin_fmaf(t, w[c][i], along);
                dw[c][i] = __builtin_fmaf(t, rstd, dw[c][i]);
            }
        }
        along = __uint_as_float(over_wave<add_f>(__float_as_uint(along)));
        const float k = rstd * rstd * (along / (float)H);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int first = (c * 64 + lane) * 8;
            if (first >= H) continue;
            float dy[8], h[8], dx[8];
            values_of<T>(dy_raw[c], dy);
            values_of<T>(h_raw[c], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) dx[i] = rstd * (dy[i] * w[c][i] - h[i] * k);
            if (a.dhidden) {
                float dh[8];
                values_of<T>(dh_raw[c], dh);
#pragma unroll
                for (int i = 0; i < 8; ++i) dx[i] += dh[i];
            }
            store_values8<T, true>(a.dX, row * a.lddx + first, 8, dx);
        }
    }
    // halves are added until one is left: wavefronts 4 - 7 to 0 - 3, 2 - 3 to 0 - 1, 1 to 0
#pragma unroll
    for (int half = kGradWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) share[wave - half][(c * 8 + i) * 64 + lane] = dw[c][i];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) dw[c][i] += share[wave][(c * 8 + i) * 64 + lane];
        }
        __syncthreads();
    }
    if (wave == 0) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int first = (c * 64 + lane) * 8;
            if (first < H) store_values8<SP24_F32, true>(a.partial, (int64_t)blockIdx.x * a.H + first, 8, dw[c]);
        }
    }
}

// out[e][c] = the sum of rows first .. last - 1 of `partial` (columns wide), in a fixed order: 32 interleaved sums, then those.
// Without offsets all rows; with them those of segment e, `unit` rows of the offsets to one of partial.
// Bound by latency: a workgroup to 32 columns is 32 of 256 units at 1024, each with 16 rows a stream one behind the other (512 x 1024 floats
// 3.8 us, 64 x 4096 4.9).
__global__ __launch_bounds__(1024) void k_column_sums(const float* partial, int64_t rows, int64_t columns, const int32_t* offsets, int unit,
                                                      float* out, unsigned from)
{
    __shared__ float part[32][33];
    const int at = threadIdx.x & 31, stream = threadIdx.x >> 5;
    const int64_t c = ((int64_t)from + blockIdx.x) * 32 + at;
    int64_t first = 0, last = rows;
    if (offsets) {
        first = min(max((int64_t)offsets[blockIdx.y] / unit, (int64_t)0), rows);
        last = min(max((int64_t)offsets[blockIdx.y + 1] / unit, first), rows);
    }
    float sum = 0.0f;
    if (c < columns) {
        int64_t i = first + stream;
        for (; i + 96 < last; i += 128) {                         // four loads on their way
            const float v0 = partial[i * columns + c], v1 = partial[(i + 32) * columns + c], v2 = partial[(i + 64) * columns + c],
                        v3 = partial[(i + 96) * columns + c];
            sum = (((sum + v0) + v1) + v2) + v3;
        }
        for (; i < last; i += 32) sum += partial[i * columns + c];
    }
    part[stream][at] = sum;
    __syncthreads();
    if (stream == 0 && c < columns) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) sum += part[i][at];
        out[(int64_t)blockIdx.y * columns + c] = sum;
    }
}

constexpr int64_t kLongRow = 32768;                               // what 1024 threads hold at four chunks each

// threads for rows of H values at C chunks a thread, in whole wavefronts
static unsigned row_threads(int64_t H, int C) { return (unsigned)(((H + 7) / 8 + C - 1) / C + 63) / 64 * 64; }

// Few rows: as many threads to a row as it has chunks, so that it is on its way at once.  Many: a few chunks a thread, so that the
// reduction (and the barrier in it) is over fewer wavefronts.
template <int T, int OUT, bool NORM>
static sp24_status run_norm(const RowsArgs& a, hipStream_t st)
{
    const bool whole = a.H % 8 == 0, many = a.N >= 1024;
    auto run = [&](auto kernel, unsigned threads) {
        const int64_t most = (1 << 21) / threads;                 // twice what the chip holds at a time
        kernel<<<(unsigned)(a.N < most ? a.N : most), threads, 0, st>>>(a);
        return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
    };
    if (!whole && many && a.H > 512 && a.H <= 4096) return run(k_norm_rows<T, OUT, 2, NORM, false, 256>, row_threads(a.H, 2));
    if (whole && many && a.H > 512 && a.H <= 4096) return run(k_norm_rows<T, OUT, 2, NORM, true, 256>, row_threads(a.H, 2));
    if (whole && many && a.H > 4096 && a.H <= 8192) return run(k_norm_rows<T, OUT, 4, NORM, true, 256>, row_threads(a.H, 4));
    if (a.H <= 8192) {
        if (whole) return run(k_norm_rows<T, OUT, 1, NORM, true, 1024>, row_threads(a.H, 1));
        return run(k_norm_rows<T, OUT, 1, NORM, false, 1024>, row_threads(a.H, 1));
    }
    if (a.H <= 16384) {
        if (whole) return run(k_norm_rows<T, OUT, 2, NORM, true, 1024>, row_threads(a.H, 2));
        return run(k_norm_rows<T, OUT, 2, NORM, false, 1024>, row_threads(a.H, 2));
    }
    if (a.H <= kLongRow) return run(k_norm_rows<T, OUT, 4, NORM, false, 1024>, row_threads(a.H, 4));
    if constexpr (!NORM) return run(k_norm_rows<T, OUT, 8, NORM, false, 1024>, row_threads(a.H, 8));
    return SP24_ERR_SHAPE;
}

template <int T>
static sp24_status run_norm_out(const RowsArgs& a, hipStream_t st)
{
    if (!a.weight) return a.out == SP24_I8 ? run_norm<T, SP24_I8, false>(a, st) : run_norm<T, SP24_F8, false>(a, st);
    switch (a.out) {
    case SP24_I8: return run_norm<T, SP24_I8, true>(a, st);
    case SP24_F8: return run_norm<T, SP24_F8, true>(a, st);
    case SP24_F32: return run_norm<T, SP24_F32, true>(a, st);
    case SP24_F16: return run_norm<T, SP24_F16, true>(a, st);
    default: return run_norm<T, SP24_BF16, true>(a, st);
    }
}

sp24_status launch_norm_rows(const RowsArgs& a, hipStream_t st)
{
    if (a.t == SP24_F32) return run_norm_out<SP24_F32>(a, st);
    if (a.t == SP24_F16) return run_norm_out<SP24_F16>(a, st);
    return run_norm_out<SP24_BF16>(a, st);
}

// rows of whole chunks that a wavefront holds
static bool short_row(int64_t H) { return H % 8 == 0 && H <= 1024; }

int64_t norm_grad_groups(int64_t N, int64_t H)
{
    // as many workgroups as the chip holds at a time (short rows: 16 wavefronts a unit), for every one writes a row of sums
    const int64_t rows = short_row(H) ? kGradWaves : 1;
    const int64_t most = short_row(H) ? 512 : (1 << 17) / (int64_t)row_threads(H, H <= 8192 ? 1 : H <= 16384 ? 2 : 4);
    return std::min((N + rows - 1) / rows, most);
}

template <int T>
static sp24_status run_norm_grad(const NormGradArgs& a, hipStream_t st)
{
    const unsigned grid = (unsigned)norm_grad_groups(a.N, a.H);
    if (grid > 0) {
        auto run = [&](auto kernel, int C) { kernel<<<grid, row_threads(a.H, C), 0, st>>>(a); };
        auto run_short = [&](auto kernel) { kernel<<<grid, 64 * kGradWaves, 0, st>>>(a); };
        if (short_row(a.H) && a.H <= 512) run_short(k_norm_grad_short<T, 1>);
        else if (short_row(a.H)) run_short(k_norm_grad_short<T, 2>);
        else if (a.H > 16384) run(k_norm_grad<T, 4, false, 1024>, 4);
        else if (a.H > 8192) run(k_norm_grad<T, 2, false, 1024>, 2);
        else if (a.H % 8 != 0) run(k_norm_grad<T, 1, false, 1024>, 1);
        else run(k_norm_grad<T, 1, true, 1024>, 1);
        if (hipGetLastError() != hipSuccess) return SP24_ERR_LAUNCH;
    }
    return launch_column_sums(a.partial, grid, a.H, nullptr, 1, 1, a.dweight, st);
}

sp24_status launch_norm_grad(const NormGradArgs& a, hipStream_t st)
{
    if (a.t == SP24_F32) return run_norm_grad<SP24_F32>(a, st);
    if (a.t == SP24_F16) return run_norm_grad<SP24_F16>(a, st);
    return run_norm_grad<SP24_BF16>(a, st);
}

sp24_status launch_column_sums(const float* partial, int64_t rows, int64_t columns, const int32_t* offsets, int segments, int unit, float* out,
                               hipStream_t st)
{
    return launch_in_parts((columns + 31) / 32, 1024, [&](unsigned from, unsigned grid) {
        k_column_sums<<<dim3(grid, (unsigned)segments), 1024, 0, st>>>(partial, rows, columns, offsets, unit, out, from);
    });
}

} // namespace sp24
