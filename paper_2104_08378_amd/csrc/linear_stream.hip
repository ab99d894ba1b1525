// Layers with few tokens, and the rows of experts that have few each, on the kernel that splits K across a workgroup's wavefronts.
// 8192 x 8192 with bias and residual, weights from HBM: 16 tokens bf16 18.3 us (76 MB at 4.2 TB/s), 14.3 where the last-level cache still has them;
// int8 and 8-bit floats 11.9 (43 MB at 3.6), one token 11.1, 64 tokens 19.2.
#include "linear.hpp"
#include "mm_stream.hpp"

namespace sp24 {

template <int DT, int BR, int NW, int NS, class ARGS>
static sp24_status run_layer_stream(const ARGS& a, hipStream_t st)
{
    const int64_t tiles_m = (a.M + 31) / 32;
    int64_t tiles_n;
    if constexpr (std::is_same<ARGS, GroupedArgs>::value) tiles_n = grouped_tiles(a.N, a.experts, BR);
    else tiles_n = (a.N + BR - 1) / BR;
    return launch_tiles(tiles_m * tiles_n, 1, 64 * NW, [&](dim3 grid, dim3 block) {
        k_spmm_stream<DT, BR, NW, NS, false, ARGS><<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n);
    });
}

sp24_status launch_linear_stream(const LinearArgs& a, hipStream_t st)
{
    return by_input(a, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const int columns = stream_columns(a);
        if (columns == 16) return run_layer_stream<DT, 16, 8, 4>(a, st);
        if (columns == 32) return run_layer_stream<DT, 32, 8, 3>(a, st);
        return run_layer_stream<DT, 64, 7, 2>(a, st);
    });
}

sp24_status launch_grouped_stream(const GroupedArgs& a, hipStream_t st)
{
    return by_input(a, [&](auto dt) { return run_layer_stream<decltype(dt)::value, 16, 8, 4>(a, st); });
}

} // namespace sp24
