// Layers on the tiled kernels: which tile takes what.
#pragma once
#include "linear.hpp"

namespace sp24 {

template <int DT, int WM, int WN, int TM, int TN, int NS, class ARGS>
static sp24_status run_layer(const ARGS& a, hipStream_t st)
{
    constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN;
    const int64_t tiles_m = (a.M + BM - 1) / BM;
    int64_t tiles_n;
    if constexpr (std::is_same<ARGS, GroupedArgs>::value) tiles_n = grouped_tiles(a.N, a.experts, BN);
    else tiles_n = (a.N + BN - 1) / BN;
    k_spmm_pipe<DT, SP24_F32, WM, WN, TM, TN, NS, 0, ARGS><<<(unsigned)(tiles_m * tiles_n), 64 * WM * WN, 0, st>>>(a, (int)tiles_m, (int)tiles_n);
    return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
}

// The lines are those of the plain product (pick_tile_general), whose loop this is.
template <int DT>
sp24_status linear_tiled(const LinearArgs& a, hipStream_t st)
{
    const int64_t cols = (a.N + 127) / 128, small = ((a.M + 127) / 128) * cols, tall = ((a.M + 255) / 256) * cols;
    const int64_t steps = a.K * (is8<DT> ? 1 : 2) / kRowBytes;
    if (small > 256 && ((a.M + 191) / 192) * cols <= 256 && steps >= 12) return run_layer<DT, 3, 2, 2, 2, 5>(a, st);
    if (small > 256 && tall <= 256 && steps >= 12) return run_layer<DT, 4, 2, 2, 2, 4>(a, st);
    const int64_t big = ((a.M + 255) / 256) * ((a.N + 255) / 256);
    const double cover_big = (double)(((a.M + 255) / 256) * 256) * (double)(((a.N + 255) / 256) * 256);
    const double cover_small = (double)(((a.M + 127) / 128) * 128) * (double)(((a.N + 127) / 128) * 128);
    if (big >= 129 && cover_big <= 1.35 * cover_small) return run_layer<DT, 4, 2, 2, 4, 3>(a, st);
    if (small <= 128) {
        if (a.N <= 64) return run_layer<DT, 2, 1, 1, 2, 9>(a, st);
        if (a.layout == SP24_LAYOUT_CANONICAL) return run_layer<DT, 2, 2, 1, 2, 7>(a, st);
        return run_layer<DT, 4, 1, 1, 2, 8>(a, st);
    }
    if (small <= 256) return run_layer<DT, 2, 2, 2, 2, 6>(a, st);
    return run_layer<DT, 2, 2, 2, 2, 3>(a, st);
}

// Rows of experts: the width that their average segment fills.
template <int DT>
sp24_status grouped_tiled(const GroupedArgs& a, hipStream_t st)
{
    const int64_t rows = a.N / a.experts;                        // a segment's, on average
    if (rows <= 64) return run_layer<DT, 2, 1, 1, 2, 9>(a, st);
    if (rows <= 512) return run_layer<DT, 2, 2, 2, 2, 3>(a, st);
    return run_layer<DT, 4, 2, 2, 4, 3>(a, st);
}

} // namespace sp24
