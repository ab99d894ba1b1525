// Argument checks shared by the C entry points; host only.
#pragma once
#include "common.hpp"

namespace sp24 {

inline bool is_input_type(sp24_dtype t) { return t == SP24_F16 || t == SP24_BF16 || t == SP24_I8 || t == SP24_F8; }
inline bool is_layout(sp24_layout l) { return l == SP24_LAYOUT_CANONICAL || l == SP24_LAYOUT_TILED; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Dimension rule of Sec. 3.2 / Sec. 4.2 on the inner dimension.
inline bool k_legal(int64_t K, sp24_dtype t) { return K > 0 && K % (esize_of(t) == 1 ? 32 : 16) == 0; }

inline bool layout_fits(int64_t M, int64_t K, sp24_layout l)
{
    return l == SP24_LAYOUT_CANONICAL || (M % 32 == 0 && K % 64 == 0);
}

inline bool out_legal(sp24_dtype in, sp24_dtype out, bool scaled)
{
    if (scaled) return in == SP24_I8 && (out == SP24_I8 || out == SP24_F32 || out == SP24_F16 || out == SP24_BF16);
    if (in == SP24_I8) return out == SP24_I32;
    return out == SP24_F32 || out == SP24_F16 || out == SP24_BF16;
}

// a matrix of `rows` rows, `cols` used columns, leading dimension ld (elements of size es);
// vec16: rows must start on 16-byte boundaries (the streaming kernels use 16-byte accesses),
// otherwise natural element alignment is enough.
inline sp24_status check_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int es, bool vec16 = true)
{
    if (rows == 0) return SP24_OK;
    if (!p) return SP24_ERR_NULL;
    if (ld < cols) return SP24_ERR_SHAPE;
    if (vec16 ? (!aligned16(p) || (ld * es) % 16 != 0) : (reinterpret_cast<uintptr_t>(p) % es != 0)) return SP24_ERR_ALIGN;
    return SP24_OK;
}

inline bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb)
{
    uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

} // namespace sp24
