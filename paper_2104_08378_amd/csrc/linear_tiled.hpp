// Layers on the tiled kernels, and on those that stage X through registers, compiled per input type.
#pragma once
#include "linear.hpp"
#include "mm_staged.hpp"

namespace sp24 {

template <int DT, int WM, int WN, int TM, int TN, int NS, class ARGS>
static sp24_status run_layer(const ARGS& a, hipStream_t st)
{
    constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN;
    const int64_t tiles_m = (a.M + BM - 1) / BM;
    int64_t tiles_n;
    if constexpr (std::is_same<ARGS, GroupedArgs>::value) tiles_n = grouped_tiles(a.N, a.experts, BN);
    else tiles_n = (a.N + BN - 1) / BN;
    return launch_tiles(tiles_m * tiles_n, 1, 64 * WM * WN, [&](dim3 grid, dim3 block) {
        k_spmm_pipe<DT, SP24_F32, WM, WN, TM, TN, NS, 0, ARGS><<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n);
    });
}

template <int DT, class ARGS>
sp24_status layer_tiled(const ARGS& a, LayerTile tile, hipStream_t st)
{
    switch (tile) {
    case LayerTile::t64x32: return run_layer<DT, 2, 1, 1, 1, 4>(a, st);
    case LayerTile::t128x64: return run_layer<DT, 4, 1, 1, 2, 4>(a, st);
    case LayerTile::t128x128: return run_layer<DT, 4, 2, 1, 2, 3>(a, st);
    case LayerTile::t128x128_one:
        if constexpr (!std::is_same<ARGS, GroupedArgs>::value) return run_layer<DT, 2, 2, 2, 2, 6>(a, st);
        return SP24_ERR_LAUNCH;
    case LayerTile::t256x128:
        if constexpr (!std::is_same<ARGS, GroupedArgs>::value) return run_layer<DT, 4, 2, 2, 2, 4>(a, st);
        return SP24_ERR_LAUNCH;                                  // (neither is a choice for experts' rows)
    default: return run_layer<DT, 4, 2, 2, 4, 3>(a, st);
    }
}

// Rows of X at any address, any legal K.  The tiles are those of the plain product there (its lines in run_staged_from).
template <int DT, class ARGS>
sp24_status layer_staged(const ARGS& a, hipStream_t st)
{
    auto run = [&](auto kernel, int bm, int bn) {
        const int64_t tiles_m = (a.M + bm - 1) / bm;
        int64_t tiles_n;
        if constexpr (std::is_same<ARGS, GroupedArgs>::value) tiles_n = grouped_tiles(a.N, a.experts, bn);
        else tiles_n = (a.N + bn - 1) / bn;
        return launch_tiles(tiles_m * tiles_n, 1, 256, [&](dim3 grid, dim3 block) { kernel<<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n); });
    };
    if (((a.M + 63) / 64) * ((a.N + 63) / 64) <= 256) return run(k_spmm_staged<DT, 0, 2, 2, 1, 1, ARGS>, 64, 64);
    if (a.M <= 64 || ((a.M + 127) / 128) * ((a.N + 127) / 128) < 256) return run(k_spmm_staged<DT, 0, 2, 2, 1, 2, ARGS>, 64, 128);
    return run(k_spmm_staged<DT, 0, 2, 2, 2, 2, ARGS>, 128, 128);
}

} // namespace sp24
