// Which products k_spmm_stream takes, and in which form.
#include "mm_stream.hpp"

namespace sp24 {

template <int DT, bool NMAJ>
static sp24_status run_stream(const MmArgs& a, hipStream_t st)
{
    const int br = stream_columns(a);
    auto run = [&](auto kernel, int nw) {
        const int tiles_m = (int)((a.M + 31) / 32), tiles_n = (int)((a.N + br - 1) / br);
        kernel<<<dim3((unsigned)(tiles_m * tiles_n), (unsigned)(a.k_slices > 1 ? a.k_slices : 1)), dim3(64 * nw), 0, st>>>(a, tiles_m, tiles_n);
        return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
    };
    // As many wavefronts as the LDS holds with two or more stages each.  Eight of 4 (N <= 16) and 3 stages (N <= 32) are
    // ahead of 16 x 2, 10 x 3, 12 x 2, 6 x 4 and 4 x 8 by 1 - 20 %; for 64 columns 7 x 2 of 5 x 3, 4 x 3 and 3 x 5 by 1 - 15 %
    if (br == 16) return run(k_spmm_stream<DT, 16, 8, 4, NMAJ>, 8);
    if (br == 32) return run(k_spmm_stream<DT, 32, 8, 3, NMAJ>, 8);
    return run(k_spmm_stream<DT, 64, 7, 2, NMAJ>, 7);
}

sp24_status launch_mm_stream(const MmArgs& a, hipStream_t st, bool* handled)
{
    *handled = false;
    const int es = esize_of(a.in);
    const bool nmajor = a.bo == SP24_B_NMAJOR;
    bool ok = a.sparse && !a.conv.on && (reinterpret_cast<uintptr_t>(a.B) & 15u) == 0 && (a.ldb * es) % 16 == 0 && (!nmajor || a.N * es % 16 == 0) &&
              a.M <= ((int64_t)1 << 30) && a.N <= ((int64_t)1 << 30) && ((a.M + 31) / 32) * ((a.N + 15) / 16) < ((int64_t)1 << 30) &&
              a.K <= ((int64_t)1 << 24);                   // 32-bit offsets inside a tile: 64 rows of B (N-major: up to 128), 32 rows of values
    ok = ok && a.ldb * es < (nmajor ? (int64_t)1 << 24 : (int64_t)1 << 25);
    if (a.layout == SP24_LAYOUT_CANONICAL) ok = ok && a.K % 32 == 0;      // codes as 4-byte words
    if (!ok) return SP24_OK;
    *handled = true;
    auto run = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        return nmajor ? run_stream<DT, true>(a, st) : run_stream<DT, false>(a, st);
    };
    if (a.in == SP24_I8) return run(std::integral_constant<int, SP24_I8>{});
    if (a.in == SP24_F8) return run(std::integral_constant<int, SP24_F8>{});
    if (a.in == SP24_F16) return run(std::integral_constant<int, SP24_F16>{});
    return run(std::integral_constant<int, SP24_BF16>{});
}

} // namespace sp24
