// Rows kept in 8 bits with a scale for every block of 128 values: what the kernels that read and write them share.
#pragma once
#include "rowops.hpp"

namespace sp24 {

template <int CODE> constexpr float kept_top() { return CODE == SP24_I8 ? 127.0f : 448.0f; }

// four values of the codes in a word, as numbers
template <int CODE>
__device__ __forceinline__ void code_values4(uint32_t w, float (&v)[4])
{
    if constexpr (CODE == SP24_I8) {
        // 2^23 + (code + 128) as its bits, a byte moved into the low end of a constant; the difference is exact.  (A conversion of an integer costs as much as
        // four of these.)
        const uint32_t u = w ^ 0x80808080u;
        v[0] = __uint_as_float(__builtin_amdgcn_perm(0x4B000000u, u, 0x07060500u)) - 8388736.0f;
        v[1] = __uint_as_float(__builtin_amdgcn_perm(0x4B000000u, u, 0x07060501u)) - 8388736.0f;
        v[2] = __uint_as_float(__builtin_amdgcn_perm(0x4B000000u, u, 0x07060502u)) - 8388736.0f;
        v[3] = __uint_as_float(__builtin_amdgcn_perm(0x4B000000u, u, 0x07060503u)) - 8388736.0f;
    } else {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1];
    }
}

// eight codes at any address, the first `n` of them; the others are zeros
template <bool WHOLE>
__device__ __forceinline__ uint2v load_codes8(const uint8_t* at, int n)
{
    if (WHOLE || n >= 8) return load_from<uint2v>(at);
    uint2v q = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) q[i / 4] |= (uint32_t)at[i] << (8 * (i % 4));
    return q;
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes8(uint8_t* at, int n, const uint2v& q)
{
    if (WHOLE || n >= 8) {
        store_to(at, q);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) at[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
}

// what eight codes stand for
template <int CODE>
__device__ __forceinline__ void kept_values8(const uint2v& q, float scale, float (&v)[8])
{
    float lo[4], hi[4];
    code_values4<CODE>(q[0], lo);
    code_values4<CODE>(q[1], hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = lo[i] * scale;
        v[i + 4] = hi[i] * scale;
    }
}

} // namespace sp24
