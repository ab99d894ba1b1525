// The weights' gradient from tokens' rows: D = A^T B, A a row of M and B a row of N for every token, all tokens or segment by segment, on the dense
// kernel of the tiled products with both operands read from LDS by transposing reads.
#pragma once
#include "linear.hpp"
#include "mm_tiled.hpp"

namespace sp24 {

template <int DT, int OUT>
sp24_status gemm_tokens(const TokenArgs& a, int experts, hipStream_t st)
{
    auto run = [&](auto kernel, int rows, int columns, int threads, int images) {
        const int64_t tiles_m = (a.M + rows - 1) / rows, tiles_n = (a.N + columns - 1) / columns;
        return launch_tiles(tiles_m * tiles_n, images, threads, [&](dim3 grid, dim3 block) { kernel<<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n); });
    };
    // K split: partial products of 128 x 128 tiles, a slice of the tokens each, in binary32
    if (a.k_slices > 1) {
        if constexpr (OUT == SP24_F32) {
            // (eight wavefronts of 64 x 32 while units are left, as below)
            const int64_t groups = ((a.M + 127) / 128) * ((a.N + 127) / 128) * a.k_slices;
            if (groups <= 176) return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 1, 4, 2, TokenArgs>, 128, 128, 512, a.k_slices);
            return run(k_gemm_pipe<DT, OUT, 2, 2, 2, 2, 4, 2, TokenArgs>, 128, 128, 256, a.k_slices);
        } else return SP24_ERR_LAUNCH;
    }
    const int64_t cols = (a.N + 127) / 128, small = ((a.M + 127) / 128) * cols, tall = ((a.M + 255) / 256) * cols, big = ((a.M + 255) / 256) * ((a.N + 255) / 256);
    const bool covered = (double)big * 256 * 256 <= 1.35 * (double)small * 128 * 128;
    // Segments, which the router makes of any length: the longest one's tiles end last, so tiles of 256 x 256, whose longest takes twice as long, are a tenth faster
    // where all are alike and a third slower where not.  us, restoring included, eight of 2048 x 1024 from 8192 choices, alike and the longest 1.6 and 3 times the
    // mean: 256 x 256 46, 61, 73; 128 x 256 50, 50, 50; 128 x 128 58, 56, 56; 64 of 1024 x 512 from 16384, alike and not: 47 and 60 to 84, 50 and 52 to 65.  (The longest
    // first: 0.98 to 1.02 times as long with eight, 0.85 with 64 uneven ones, 1.0 to 1.08 with even ones.)
    // Few tiles: half as large ones, four stages deep.  Eight of 512 x 512 from 8192 24.5 -> 19.5, uneven 41 -> 29; eight of 1024 x 512 24.6 -> 22.9, 40 -> 30;
    // four of 1024 x 1024 34.1 -> 33.6, 40 -> 36; but (256 tiles) 16 of 1024 x 512 from 1024 10.5 -> 12.4.  Columns of 128 too where wider ones are mostly padding,
    // and where segments are short, two workgroups to a unit then, one's first transfers and results beside the other's products: eight of 4096 x 2048 from 512 choices
    // 48.9 -> 46.0, uneven 47.5 -> 44.6; 16 of 1344 x 1472 from 94 26.0 -> 22.2; eight of 4096 x 1024 from 1024 32.7 -> 31.9; 16 of 1024 x 1024 from 2048 20.0 -> 21.3.
    if (a.offsets) {
        const int64_t wide = (a.N + 255) / 256;
        if ((a.M + 127) / 128 * wide * experts <= 128) return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 1, 4, 2, TokenArgs>, 128, 128, 512, experts);
        if (wide * 256 * 4 > cols * 128 * 5 || a.K <= 128 * experts) return run(k_gemm_pipe<DT, OUT, 4, 2, 1, 2, 2, 2, TokenArgs>, 128, 128, 512, experts);
        return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 2, 3, 2, TokenArgs>, 128, 256, 512, experts);
    }
    // All tokens: the tile whose workgroups still find a unit each, as for the product of an M x K operand (us, restoring included): 512 x 512 x 8192 on 64 x 64
    // 41.2, 128 x 64 47.7, 128 x 128 51.3; 2048 x 1024 x 4096 on 64 x 64 37.6, 128 x 64 30.5, 128 x 128 32.6; 4096 x 1024 x 8192 on 128 x 128, four wavefronts 79.9,
    // eight 82.1, 256 x 128 94.3; 8192 x 2048 x 2048 on 256 x 256 65.8, 256 x 128 69.1, 128 x 128 76.2.
    // Four stages: 640 x 1000 x 509 with two to five and nine 9.9, 8.7, 8.5, 8.7, 9.8; 768 x 768 x 2048 21.3, 15.0, 13.9, 14.2, 15.0; on 128 x 64 1024 x 1024 x 1024 with
    // two to six 13.3, 10.5, 10.0, 10.2, 11.1: transfers ahead of what a short K has cost their time before the first product.
    if (small <= 64) return run(k_gemm_pipe<DT, OUT, 2, 2, 1, 1, 4, 2, TokenArgs>, 64, 64, 256, 1);
    if (small <= 128) return run(k_gemm_pipe<DT, OUT, 4, 1, 1, 2, 4, 2, TokenArgs>, 128, 64, 256, 1);
    if (small <= 176) return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 1, 4, 2, TokenArgs>, 128, 128, 512, 1);
    if (small <= 256) return run(k_gemm_pipe<DT, OUT, 2, 2, 2, 2, 4, 2, TokenArgs>, 128, 128, 256, 1);
    if (tall <= 256) return run(k_gemm_pipe<DT, OUT, 4, 2, 2, 2, 3, 2, TokenArgs>, 256, 128, 512, 1);
    if (big >= 129 && covered) return run(k_gemm_pipe<DT, OUT, 4, 2, 2, 4, 2, 2, TokenArgs>, 256, 256, 512, 1);
    return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 2, 3, 2, TokenArgs>, 128, 256, 512, 1);
}

} // namespace sp24
