// What the kernels around the products share: values of rows in binary32, activations, sums over a wavefront.
#pragma once
#include "common.hpp"

namespace sp24 {

typedef float float4v __attribute__((ext_vector_type(4)));

// A value of global memory at any address that its element type allows (the chip loads and stores 16 bytes from there).
template <typename V>
__device__ __forceinline__ V load_from(const void* p)
{
    struct __attribute__((packed, aligned(1))) any_t { V v; };
    return reinterpret_cast<const any_t*>(p)->v;
}
template <typename V>
__device__ __forceinline__ void store_to(void* p, const V& v)
{
    struct __attribute__((packed, aligned(1))) any_t { V v; };
    reinterpret_cast<any_t*>(p)->v = v;
}

template <int T> constexpr int value_size() { return T == SP24_F32 ? 4 : is8<T> ? 1 : 2; }

template <int T>
__device__ __forceinline__ float value_of(uint32_t bits)
{
    if constexpr (T == SP24_F32) return __uint_as_float(bits);
    else if constexpr (T == SP24_BF16) return __uint_as_float(bits << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

template <int T>
__device__ __forceinline__ float load_value(const void* p, int64_t i)
{
    if constexpr (T == SP24_F32) return reinterpret_cast<const float*>(p)[i];
    else return value_of<T>(reinterpret_cast<const uint16_t*>(p)[i]);
}

// Eight neighbouring values as they lie in memory (the unit of work of a lane: 16 bytes of a 16-bit type), the first `n` of
// them; the others are zeros.
// (WHOLE: there are eight)
template <int T> struct raw8 { uint4v q[T == SP24_F32 ? 2 : 1]; };
template <int T, bool WHOLE = false>
__device__ __forceinline__ raw8<T> load_raw8(const void* p, int64_t first, int n)
{
    const uint8_t* at = reinterpret_cast<const uint8_t*>(p) + first * value_size<T>();
    raw8<T> r = {};
    if (WHOLE || n >= 8) {
        r.q[0] = load_from<uint4v>(at);
        if constexpr (T == SP24_F32) r.q[1] = load_from<uint4v>(at + 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (T == SP24_F32) r.q[i / 4][i % 4] = i < n ? reinterpret_cast<const uint32_t*>(at)[i] : 0u;
            else r.q[0][i / 2] |= i < n ? (uint32_t)reinterpret_cast<const uint16_t*>(at)[i] << (16 * (i & 1)) : 0u;
        }
    }
    return r;
}
template <int T>
__device__ __forceinline__ void values_of(const raw8<T>& r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (T == SP24_F32) v[i] = __uint_as_float(r.q[i / 4][i % 4]);
        else v[i] = value_of<T>((r.q[0][i / 2] >> (16 * (i & 1))) & 0xFFFFu);
    }
}

// The first `n` of eight values, rounded to nearest even.
template <int T, bool WHOLE = false>
__device__ __forceinline__ void store_values8(void* p, int64_t first, int n, const float (&v)[8])
{
    uint8_t* at = reinterpret_cast<uint8_t*>(p) + first * value_size<T>();
    if constexpr (T == SP24_F32) {
        if (WHOLE || n >= 8) {
            store_to(at, float4v{v[0], v[1], v[2], v[3]});
            store_to(at + 16, float4v{v[4], v[5], v[6], v[7]});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) reinterpret_cast<float*>(at)[i] = v[i];
        }
    } else {
        const uint4v q = {pack_out16<T>(v[0], v[1]), pack_out16<T>(v[2], v[3]), pack_out16<T>(v[4], v[5]), pack_out16<T>(v[6], v[7])};
        if (WHOLE || n >= 8) store_to(at, q);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) reinterpret_cast<uint16_t*>(at)[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
        }
    }
}

// Eight vector entries in binary32, the first `n` of them.
template <bool WHOLE = false>
__device__ __forceinline__ void load_floats8(const float* p, int64_t first, int n, float (&v)[8])
{
    values_of<SP24_F32>(load_raw8<SP24_F32, WHOLE>(p, first, n), v);
}

// ---------------------------------------------------------------------------
// Activations of a product's epilogue, in binary32: p = 1 / (1 + e^-x) by the chip's own 2^x and reciprocal (1 ulp each), and
//   silu(z) = z p(z),  gelu(z) = z p(2u) with u = sqrt(2/pi) (z + 0.044715 z^3), which is the tanh form, for 1 + tanh u = 2 p(2u).
// ---------------------------------------------------------------------------
constexpr float kLog2e = 1.442695040888963f, kGelu2C = 1.5957691216057308f;         // 2 sqrt(2 / pi)

// from t = -x log2(e)
__device__ __forceinline__ float logistic_of(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t)); }
__device__ __forceinline__ float logistic(float x) { return logistic_of(-kLog2e * x); }
// p(2u), from z and z^2
__device__ __forceinline__ float logistic_2u(float z, float square)
{
    return logistic_of(z * __builtin_fmaf(-0.044715f * kGelu2C * kLog2e, square, -kGelu2C * kLog2e));
}

template <int ACT>
__device__ __forceinline__ float activated(float z)
{
    if constexpr (ACT == SP24_ACT_RELU) return z > 0.0f || z != z ? z : 0.0f;        // (a NaN stays one)
    else if constexpr (ACT == SP24_ACT_GELU) return z * logistic_2u(z, z * z);
    else if constexpr (ACT == SP24_ACT_SILU) return z * logistic(z);
    else return z;
}

// (one branch for all of them: `act` is the same in every lane)
template <int COUNT>
__device__ __forceinline__ void activate(float (&v)[COUNT], int act)
{
    auto all = [&](auto f) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = f(v[i]);
    };
    if (act == SP24_ACT_GELU) all([](float z) { return activated<SP24_ACT_GELU>(z); });
    else if (act == SP24_ACT_SILU) all([](float z) { return activated<SP24_ACT_SILU>(z); });
    else if (act == SP24_ACT_RELU) all([](float z) { return activated<SP24_ACT_RELU>(z); });
}

// d activate / d z.  Past |z| = 100 the slopes are 0 and 1 (p is 0 or 1): the factors beside p (1 - p) are held where they stay finite.  (A
// NaN goes through p.)
__device__ __forceinline__ float activation_slope(float z, int act)
{
    if (act == SP24_ACT_RELU) return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    const float x = __builtin_amdgcn_fmed3f(z, -100.0f, 100.0f);
    if (act == SP24_ACT_GELU) {
        const float square = __builtin_fminf(z * z, 1e4f);
        const float p = logistic_2u(z, square);
        return __builtin_fmaf(x * __builtin_fmaf(0.134145f * kGelu2C, square, kGelu2C), __builtin_fmaf(-p, p, p), p);
    }
    if (act == SP24_ACT_SILU) {
        const float p = logistic(z);
        return __builtin_fmaf(x, __builtin_fmaf(-p, p, p), p);
    }
    return 1.0f;
}

// ---------------------------------------------------------------------------
// Sum (largest bit pattern) over the 64 lanes, the same in all of them, always in the same order.
// ---------------------------------------------------------------------------
struct add_f { __device__ static __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); } };
struct max_u { __device__ static __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; } };
template <class OP>
__device__ __forceinline__ uint32_t over_wave(uint32_t v)
{
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));     // quad_perm [1,0,3,2]
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));     // quad_perm [2,3,0,1]
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));    // the other half of eight lanes, mirrored
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));    // the other half of sixteen
    v = OP::of(v, (uint32_t)__shfl_xor((int)v, 16));
    return OP::of(v, (uint32_t)__shfl_xor((int)v, 32));
}

// The same over the wavefronts of a workgroup (up to 16) through `cells`, 16 words of LDS.  One barrier: a caller uses the cells again
// only behind another one.
template <class OP>
__device__ __forceinline__ uint32_t over_workgroup(uint32_t v, uint32_t* cells)
{
    v = over_wave<OP>(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) cells[threadIdx.x >> 6] = v;
    __syncthreads();
    const int i = threadIdx.x & 15;
    v = i < waves ? cells[i] : 0u;                                                             // 0: nothing, to either operation
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
    v = OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
    return OP::of(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
}

} // namespace sp24
