// The weights' gradient from tokens' rows: D = A^T B, A a row of M and B a row of N for every token, all tokens or segment by segment, on the dense
// kernel of the tiled products with both operands read from LDS by transposing reads.
#pragma once
#include "linear.hpp"
#include "mm_tiled.hpp"

namespace sp24 {

template <int DT, int OUT>
sp24_status gemm_tokens(const TokenArgs& a, int experts, hipStream_t st)
{
    auto run = [&](auto kernel, int rows, int columns, int threads) {
        const int64_t tiles_m = (a.M + rows - 1) / rows, tiles_n = (a.N + columns - 1) / columns;
        return launch_tiles(tiles_m * tiles_n, experts, threads, [&](dim3 grid, dim3 block) { kernel<<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n); });
    };
    if (a.offsets) {
        if ((a.N + 255) / 256 * 256 * 4 > (a.N + 127) / 128 * 128 * 5) return run(k_gemm_pipe<DT, OUT, 4, 2, 1, 2, 2, 2, TokenArgs>, 128, 128, 512);
        return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 2, 3, 2, TokenArgs>, 128, 256, 512);
    }
    const int64_t cols = (a.N + 127) / 128, small = ((a.M + 127) / 128) * cols, tall = ((a.M + 255) / 256) * cols, big = ((a.M + 255) / 256) * ((a.N + 255) / 256);
    const double cover_big = (double)(((a.M + 255) / 256) * 256) * (double)(((a.N + 255) / 256) * 256), cover_small = (double)small * 128 * 128;
    if (small <= 128) return run(k_gemm_pipe<DT, OUT, 4, 1, 1, 2, 6, 2, TokenArgs>, 128, 64, 256);
    if (small <= 176) return run(k_gemm_pipe<DT, OUT, 4, 2, 1, 2, 4, 2, TokenArgs>, 128, 128, 512);
    if (small <= 256) return run(k_gemm_pipe<DT, OUT, 2, 2, 2, 2, 4, 2, TokenArgs>, 128, 128, 256);
    if (tall <= 256) return run(k_gemm_pipe<DT, OUT, 4, 2, 2, 2, 3, 2, TokenArgs>, 256, 128, 512);
    if (big >= 129 && cover_big <= 1.35 * cover_small) return run(k_gemm_pipe<DT, OUT, 4, 2, 2, 4, 2, 2, TokenArgs>, 256, 256, 512);
    return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 2, 3, 2, TokenArgs>, 128, 256, 512);
}

} // namespace sp24
