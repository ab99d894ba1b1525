// Layers on the sparse product: which kernel takes what.
#include <algorithm>
#include <cmath>

#include "linear.hpp"

namespace sp24 {

// What the kernels that transfer X into LDS ask of it: rows of 16 bytes, whole 32-byte runs and (canonical codes come as words) whole words.
static bool transferable(const LinearArgs& a)
{
    const int64_t es = esize_of(a.in);
    return (reinterpret_cast<uintptr_t>(a.B) & 15u) == 0 && (a.ldb * es) % 16 == 0 && a.ldb * es < ((int64_t)1 << 22) && a.K <= ((int64_t)1 << 24) &&
           (a.layout == SP24_LAYOUT_TILED || (a.K % 32 == 0 && a.K / 2 * es * 256 < ((int64_t)1 << 31)));
}

// Which kernel: the least of estimates of the form  base + max(steps * alone, (steps * step + tile) * workgroups / units)  in us, a step being
// 128 bytes of K: one workgroup's own time, and what the workgroups of a compute unit (several at a time, except where they come in whole
// rounds) take of it together.  Fitted to 970 layers and 1050 sets of experts' rows of 128 - 16384 rows of weights, K 256 - 8192, 1 - 16384 rows, all
// types, from HBM: within 9 - 13 % of the measured time on average, and the choice within 3.9 % of the best of twelve kernels (layers; at worst 1.5
// times) and 3.7 % (experts).  One shape throughout costs 26 % (64 x 32), 13 % (128 x 128 besides), 6 % (the streaming kernel besides).  E.g.
// bf16, us: 1664 x 1158 x 1728 10.0 on 128 x 64 and 12.8 on 128 x 128; 13275 x 2198 x 384 42 and 52; experts of 4096 x 4096 on 32 rows of eight
// segments 29.3 on 64 x 32 and 36.4 on the streaming kernel, whose workgroups come one to a unit.
// 8-bit: experts of 4096 x 4096 on 16 tokens of two each, from HBM, 18.2 (84 MB at 4.6 TB/s; bf16 28), of 4096 x 1024 on 509 tokens 14.2 (bf16 18.0); layers
// 4096 x 8192 x 1024 to bf16 with GELU int8 45.5, 8-bit floats 44.2, 11008 x 333 x 4096 with SiLU 22.2 and 22.0.
struct LayerCost {
    LayerTile tile;
    int rows, columns;
    bool whole_rounds;
    double base, alone, step, each;                             // tiled layout
    double c_base, c_alone, c_step, c_each;                     // canonical
};
constexpr LayerCost kLayerCosts[] = {
    {LayerTile::stream, 32, 16, true, 3.5, 0.034, 0.09, 0.45, 3.5, 0.05, 0.10, 0.5},
    {LayerTile::stream, 32, 32, true, 3.6, 0.042, 0.071, 0.8, 3.5, 0.056, 0.097, 1.0},
    {LayerTile::stream, 32, 64, true, 3.6, 0.114, 0.098, 2.6, 3.9, 0.111, 0.117, 2.6},
    {LayerTile::t64x32, 64, 32, false, 3.8, 0.12, 0.092, 0.74, 4.1, 0.10, 0.17, 0.48},
    {LayerTile::t128x64, 128, 64, false, 4.5, 0.16, 0.24, 2.2, 5.1, 0.19, 0.47, 1.5},
    {LayerTile::t128x128, 128, 128, false, 4.8, 0.26, 0.43, 2.4, 5.4, 0.35, 0.74, 1.0},
    {LayerTile::t128x128_one, 128, 128, true, 6.2, 0.25, 0.29, 5.3, 6.8, 0.36, 0.45, 5.7},
    {LayerTile::t256x128, 256, 128, true, 7.3, 0.32, 0.80, 1.0, 7.4, 0.57, 1.25, 1.0},
};

// workgroups(cost): of the launch, as far as the host knows
template <class F>
static LayerTile cheapest(const MmArgs& a, int stream_width, bool grouped, F&& workgroups)
{
    const double steps = (double)a.K * esize_of(a.in) / 128;
    double least = 0;
    LayerTile best = LayerTile::t64x32;
    for (const LayerCost& c : kLayerCosts) {
        if (c.tile == LayerTile::stream && c.columns != stream_width) continue;
        if (grouped && (c.tile == LayerTile::t256x128 || c.tile == LayerTile::t128x128_one)) continue;
        const bool canonical = a.layout == SP24_LAYOUT_CANONICAL;
        double units = workgroups(c) / 256;
        if (c.whole_rounds && units > 1) units = std::ceil(units);
        const double us = (canonical ? c.c_base : c.base) + std::max(steps * (canonical ? c.c_alone : c.alone),
                                                                      (steps * (canonical ? c.c_step : c.step) + (canonical ? c.c_each : c.each)) * units);
        if (least == 0 || us < least) {
            least = us;
            best = c.tile;
        }
    }
    return best;
}

sp24_status launch_linear(const LinearArgs& a, hipStream_t st)
{
    if (!transferable(a)) return by_input(a, [&](auto dt) { return layer_staged<decltype(dt)::value>(a, st); });
    // 256 x 256 tiles where the plain product takes them, and four steps at least (two: 24.5 - 35 us against 20 - 25 on 128 x 128)
    const int64_t big = ((a.M + 255) / 256) * ((a.N + 255) / 256);
    const double cover_big = (double)(((a.M + 255) / 256) * 256) * (double)(((a.N + 255) / 256) * 256);
    const double cover_small = (double)(((a.M + 127) / 128) * 128) * (double)(((a.N + 127) / 128) * 128);
    LayerTile tile = LayerTile::t256x256;
    if (!(big >= 129 && cover_big <= 1.35 * cover_small && a.K * esize_of(a.in) >= 4 * 128))
        tile = cheapest(a, stream_columns(a), false, [&](const LayerCost& c) { return (double)((a.M + c.rows - 1) / c.rows) * (double)((a.N + c.columns - 1) / c.columns); });
    if (tile == LayerTile::stream) return launch_linear_stream(a, st);
    return by_input(a, [&](auto dt) { return layer_tiled<decltype(dt)::value>(a, tile, st); });
}

sp24_status launch_linear_grouped(const GroupedArgs& a, hipStream_t st)
{
    if (!transferable(a)) return by_input(a, [&](auto dt) { return layer_staged<decltype(dt)::value>(a, st); });
    // The host knows the rows' number at most: a segment is taken to end in the middle of its last sixteen and of its last tile.
    const double live = (double)std::min<int64_t>(a.experts, a.N / kSegmentRows), rows = (double)a.N - 8 * live;
    auto columns = [&](int width) { return width == 16 ? (double)a.N / 16 : std::max(live, rows / width + 0.5 * live * (1 - 16.0 / width)); };
    LayerTile tile = cheapest(a, 16, true, [&](const LayerCost& c) { return (double)((a.M + c.rows - 1) / c.rows) * columns(c.columns); });
    // 256 x 256 where they make one round and have many steps: 0.84 - 0.96 of the others' time (with fewer of either up to 1.3)
    const double big = (double)((a.M + 255) / 256) * columns(256);
    if (big >= 129 && big <= 200 && a.K * esize_of(a.in) >= 24 * 128) tile = LayerTile::t256x256;
    if (tile == LayerTile::stream) return launch_grouped_stream(a, st);
    return by_input(a, [&](auto dt) { return layer_tiled<decltype(dt)::value>(a, tile, st); });
}

// The segments' dense products, A [M, rows] and B [rows, N], all segments in one launch.  Segments are short, so that a tile's first operands
// and its way out weigh as much as its steps, and a step's bytes set the pace: tiles of 128 x 256 on eight wavefronts, whose rows of B are 512 bytes
// (eight segments of 8240 rows, 2048 x 1024 bf16: 128 x 128 with four stages 52.7 us, 256 x 128 59.8, 256 x 256 64, 128 x 256 46.7; sixteen of
// 4224, 1024 x 1024 27.6, 24.5, 31.7 and 20.9), and where columns would be wasted 128 x 128, two workgroups to a unit (52.5; 25.0).
template <int DT, int OUT>
static sp24_status run_segments(const SegmentArgs& a, int experts, hipStream_t st)
{
    auto run = [&](auto kernel, int columns) {
        const int64_t tiles_m = (a.M + 127) / 128, tiles_n = (a.N + columns - 1) / columns;
        return launch_tiles(tiles_m * tiles_n, experts, 512, [&](dim3 grid, dim3 block) { kernel<<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n); });
    };
    if ((a.N + 255) / 256 * 256 * 4 > (a.N + 127) / 128 * 128 * 5) return run(k_gemm_pipe<DT, OUT, 4, 2, 1, 2, 2, 2, SegmentArgs>, 128);
    return run(k_gemm_pipe<DT, OUT, 2, 4, 2, 2, 3, 2, SegmentArgs>, 256);
}

sp24_status launch_gemm_grouped(const SegmentArgs& a, int experts, hipStream_t st)
{
    if (a.in == SP24_F16) return a.out == SP24_F32 ? run_segments<SP24_F16, SP24_F32>(a, experts, st) : run_segments<SP24_F16, SP24_F16>(a, experts, st);
    return a.out == SP24_F32 ? run_segments<SP24_BF16, SP24_F32>(a, experts, st) : run_segments<SP24_BF16, SP24_BF16>(a, experts, st);
}

} // namespace sp24
