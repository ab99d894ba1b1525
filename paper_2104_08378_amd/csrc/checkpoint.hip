// Rows kept in 8 bits for the backward pass, and had again.
//
//   m = max |x| of 128 neighbouring values, scale = m / top, code = RNE(x top / m);  again: act(code scale)
//
// Bound by memory: a 16-bit value costs 3 bytes one way and 3 the other.  Sixteen lanes hold a block, eight values each, so that its largest
// magnitude takes four exchanges of neighbouring lanes and no LDS.  8192 x 4096 bf16 from HBM: kept in 22.0 us, 101 MB at 4.6 TB/s, had again in 22 (4.6), with GELU
// 24; 16 x 8192 2.2, a launch.  From binary32, 4096 x 4096, 14 from the last-level cache.  (More rows a thread, two to eight, were 2 % faster to 20 % slower; workgroups of 512 level.)
#include "kept.hpp"
#include "launch.hpp"

namespace sp24 {

constexpr float kLeastKept = 7.888609052210118e-31f;            // 2^-100: a block below it has its codes taken against it

// row and block of row of the number `at` among rows of `blocks` blocks
__device__ __forceinline__ void place_of(int64_t at, int64_t blocks, int64_t& row, int64_t& block)
{
    if ((uint64_t)at >> 32 == 0) row = (uint32_t)at / (uint32_t)blocks;      // (one division of 32 bits where that is enough)
    else row = at / blocks;
    block = at - row * blocks;
}

template <int T, int CODE, bool WHOLE>
__global__ __launch_bounds__(256) void k_checkpoint_rows(KeepArgs a, int64_t blocks, unsigned from)
{
    int64_t row, block;
    place_of(((int64_t)from + blockIdx.x) * 16 + (threadIdx.x >> 4), blocks, row, block);
    const int64_t first = block * kKeptBlock + (threadIdx.x & 15) * 8;
    const int n = row < a.N ? (int)min(max(a.H - first, (int64_t)0), (int64_t)8) : 0;
    raw8<T> x = {};
    if (n > 0) x = load_raw8<T, WHOLE>(a.X, row * a.ldx + first, n);
    float v[8];
    values_of<T>(x, v);
    // Magnitudes go by their bit patterns, in which infinity and NaN are the largest.
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    most = max_u::of(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xF, 0xF, true));
    most = max_u::of(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xF, 0xF, true));
    most = max_u::of(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x141, 0xF, 0xF, true));
    most = max_u::of(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x140, 0xF, 0xF, true));
    const bool finite = most < 0x7F800000u;
    const float m = finite ? fmaxf(__uint_as_float(most), kLeastKept) : 1.0f;
    if (T == SP24_F32) {
        const double wide = (double)m, inv = 1.0 / wide;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double p = (double)v[i] * (double)kept_top<CODE>(), q = p * inv;
            v[i] = (float)__builtin_fma(__builtin_fma(-q, wide, p), inv, q);
        }
    } else {
        // The quotient as IEEE division rounds it, in four operations a value: x top has 18 bits at most and is exact, q is within two units of
        // the last place, the rest p - q m is exact (m has 11 bits), and what it adds to q brings the sum within 2^-23 of a unit, while no quotient of so few bits
        // lies nearer than 2^-13 to the middle between two numbers.  A power of two in front keeps all of it away from the type's ends.
        const uint32_t exponent = min(__float_as_uint(m) >> 23, 253u);
        const float power = __uint_as_float((254u - exponent) << 23), unit = m * power, inv = 1.0f / unit, t = kept_top<CODE>() * power;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = v[i] * t, q = p * inv;
            v[i] = __builtin_fmaf(__builtin_fmaf(-q, unit, p), inv, q);
        }
    }
    uint2v q = {0u, 0u};
    if (finite) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            if constexpr (CODE == SP24_I8) {
                // 1.5 2^23 more: the sum is rounded to a whole number, ties to even, whose low byte is the code
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(v[4 * d + i] + 12582912.0f);
                q[d] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0C0C0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), 0x05040100u);
            } else {
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * d], v[4 * d + 1], 0, false);
                q[d] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * d + 2], v[4 * d + 3], w, true);
            }
        }
    }
    // (Stores past the L2 are 10 % faster for 16-bit values, and what is had again soon is 20 % slower then: 8192 x 4096 kept and restored 38.3 -> 41.9 us.)
    if (n > 0) store_codes8<WHOLE>(reinterpret_cast<uint8_t*>(a.codes) + row * a.ldc + first, n, q);
    if (row < a.N && (threadIdx.x & 15) == 0) a.scale[row * blocks + block] = finite ? m / kept_top<CODE>() : __builtin_nanf("");
}

template <int T, int CODE, bool WHOLE>
__global__ __launch_bounds__(256) void k_restore_rows(RestoreArgs a, int64_t blocks, unsigned from)
{
    int64_t row, block;
    place_of(((int64_t)from + blockIdx.x) * 16 + (threadIdx.x >> 4), blocks, row, block);
    const int64_t first = block * kKeptBlock + (threadIdx.x & 15) * 8;
    const int n = (int)min(a.H - first, (int64_t)8);
    if (row >= a.R || n <= 0) return;
    int64_t token = row;
    if (a.rows) {
        const int choice = a.rows[row];
        token = choice < 0 ? -1 : choice / a.topk;
    }
    float v[8] = {};
    if (token >= 0 && token < a.N) {
        const uint2v q = load_codes8<WHOLE>(reinterpret_cast<const uint8_t*>(a.codes) + token * a.ldc + first, n);
        kept_values8<CODE>(q, a.scale[token * blocks + block], v);
        activate(v, a.act);
    }
    store_values8<T, WHOLE>(a.out, row * a.ldo + first, n, v);
}

// f(integral_constant<int, t>{}) for a float type, f(integral_constant<int, code>{}) for an 8-bit one
template <class F>
static void by_float(sp24_dtype t, F&& f)
{
    if (t == SP24_F32) f(std::integral_constant<int, SP24_F32>{});
    else if (t == SP24_F16) f(std::integral_constant<int, SP24_F16>{});
    else f(std::integral_constant<int, SP24_BF16>{});
}
template <class F>
static void by_code(sp24_dtype t, F&& f)
{
    if (t == SP24_I8) f(std::integral_constant<int, SP24_I8>{});
    else f(std::integral_constant<int, SP24_F8>{});
}

sp24_status launch_checkpoint_rows(const KeepArgs& a, hipStream_t st)
{
    const int64_t blocks = kept_blocks(a.H);
    return launch_in_parts((a.N * blocks + 15) / 16, 256, [&](unsigned from, unsigned grid) {
        by_float(a.t, [&](auto t) {
            by_code(a.code, [&](auto c) {
                constexpr int T = decltype(t)::value, C = decltype(c)::value;
                if (a.H % 8 == 0) k_checkpoint_rows<T, C, true><<<grid, 256, 0, st>>>(a, blocks, from);
                else k_checkpoint_rows<T, C, false><<<grid, 256, 0, st>>>(a, blocks, from);
            });
        });
    });
}

sp24_status launch_restore_rows(const RestoreArgs& a, hipStream_t st)
{
    const int64_t blocks = kept_blocks(a.H);
    return launch_in_parts((a.R * blocks + 15) / 16, 256, [&](unsigned from, unsigned grid) {
        by_float(a.t, [&](auto t) {
            by_code(a.code, [&](auto c) {
                constexpr int T = decltype(t)::value, C = decltype(c)::value;
                if (a.H % 8 == 0) k_restore_rows<T, C, true><<<grid, 256, 0, st>>>(a, blocks, from);
                else k_restore_rows<T, C, false><<<grid, 256, 0, st>>>(a, blocks, from);
            });
        });
    });
}

} // namespace sp24
