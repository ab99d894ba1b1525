// Layers on the sparse product: the kernel for operands at any alignment, and which kernel takes what.
#include <algorithm>

#include "linear.hpp"

namespace sp24 {

// One wavefront to 32 features and 32 tokens, operands straight from memory: any legal K, X at any address.
template <int DT, class ARGS>
__global__ __launch_bounds__(64) void k_linear_any(ARGS a, int tiles_m)
{
    constexpr int ES = is8<DT> ? 1 : 2;
    constexpr int TB = 64 * ES;                              // bytes of a row of X per 64-column tile
    const int lane = threadIdx.x, r = lane & 31, q = lane >> 5;
    const int tm = blockIdx.x % tiles_m;
    int tn = blockIdx.x / tiles_m;
    if (!a.template enter<32, 32>(tm, tn)) return;
    const int64_t m0 = (int64_t)tm * 32;
    const int64_t n = (int64_t)tn * 32 + r;
    const uint8_t* x = reinterpret_cast<const uint8_t*>(a.B) + min(n, a.N - 1) * a.ldb * ES;
    compressed_rows<DT, 1> rows;
    rows.init(a, tm, lane);
    typename acc_of<DT>::type acc = {};
    const int64_t Kbytes = a.K * ES;
    for (int64_t kb = 0; kb * 64 < a.K; ++kb) {
        int4v v[1][rows.NA];
        uint32_t code[1];
        if (kb * 64 + 64 <= a.K) rows.load_whole(kb, v, code);
        else rows.load_edge(kb, v, code);
        uint4v piece[TB / 32];                               // this lane's 16 bytes of every 32 (K is whole 32-byte runs)
#pragma unroll
        for (int p = 0; p < TB / 32; ++p) {
            const int64_t off = kb * TB + 32 * p + 16 * q;
            piece[p] = off < Kbytes ? load16_any(x + off) : uint4v{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int j = 0; j < rows.NA; ++j) {
            const uint4v lo = is8<DT> ? piece[0] : piece[j], hi = is8<DT> ? piece[1] : piece[2 + j];
            int8v f;
            f[0] = lo[0]; f[1] = lo[1]; f[2] = lo[2]; f[3] = lo[3];
            f[4] = hi[0]; f[5] = hi[1]; f[6] = hi[2]; f[7] = hi[3];
            if (j == 0) acc = smfmac32<DT, 0>(v[0][0], f, acc, (int)code[0]);
            else acc = smfmac32<DT, 1>(v[0][rows.NA - 1], f, acc, (int)code[0]);
        }
    }
    if (n >= a.N) return;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int64_t m = m0 + 8 * g + 4 * q;
        if (m >= a.M) continue;
        typename LinearArgs::template way_out<DT, 4> out;
        out.fetch(a, n, m);
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (float)acc[4 * g + i];
        out.finish(a, n, m, y);
    }
}

template <class F>
static sp24_status by_input(const MmArgs& a, F&& run)
{
    if (a.in == SP24_I8) return run(std::integral_constant<int, SP24_I8>{});
    if (a.in == SP24_F8) return run(std::integral_constant<int, SP24_F8>{});
    if (a.in == SP24_F16) return run(std::integral_constant<int, SP24_F16>{});
    return run(std::integral_constant<int, SP24_BF16>{});
}

template <class ARGS>
static sp24_status run_any(const ARGS& a, int64_t tiles_n, hipStream_t st)
{
    const int64_t tiles_m = (a.M + 31) / 32;
    return by_input(a, [&](auto dt) {
        k_linear_any<decltype(dt)::value, ARGS><<<(unsigned)(tiles_m * tiles_n), 64, 0, st>>>(a, (int)tiles_m);
        return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
    });
}

// What the kernels that transfer X into LDS ask of it: rows of 16 bytes, whole 32-byte runs and (canonical codes come as words) whole words.
static bool transferable(const LinearArgs& a)
{
    const int64_t es = esize_of(a.in);
    return (reinterpret_cast<uintptr_t>(a.B) & 15u) == 0 && (a.ldb * es) % 16 == 0 && a.ldb * es < ((int64_t)1 << 22) && a.K <= ((int64_t)1 << 24) &&
           (a.layout == SP24_LAYOUT_TILED || (a.K % 32 == 0 && a.K / 2 * es * 256 < ((int64_t)1 << 31)));
}

sp24_status launch_linear(const LinearArgs& a, hipStream_t st)
{
    if (!transferable(a)) return run_any(a, (a.N + 31) / 32, st);
    const int64_t tiles = (a.M + 127) / 128;
    if (stream_workgroups(a) <= 256 || (a.N <= 32 && tiles < 86)) return launch_linear_stream(a, st);
    return by_input(a, [&](auto dt) { return linear_tiled<decltype(dt)::value>(a, st); });
}

sp24_status launch_linear_grouped(const GroupedArgs& a, hipStream_t st)
{
    if (!transferable(a)) return run_any(a, grouped_tiles(a.N, a.experts, 32), st);
    if (a.N <= 32 * (int64_t)a.experts) return launch_grouped_stream(a, st);
    return by_input(a, [&](auto dt) { return grouped_tiled<decltype(dt)::value>(a, st); });
}

// The segments' dense products, A [M, rows] and B [rows, N]: 128 x 128 tiles, all segments in one launch.
template <int DT, int OUT>
static sp24_status run_segments(const SegmentArgs& a, int experts, hipStream_t st)
{
    const int tiles_m = (int)((a.M + 127) / 128), tiles_n = (int)((a.N + 127) / 128);
    k_gemm_pipe<DT, OUT, 2, 2, 2, 2, 4, 2, SegmentArgs><<<dim3((unsigned)(tiles_m * tiles_n), (unsigned)experts), 256, 0, st>>>(a, tiles_m, tiles_n);
    return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
}

sp24_status launch_gemm_grouped(const SegmentArgs& a, int experts, hipStream_t st)
{
    if (a.in == SP24_F16) return a.out == SP24_F32 ? run_segments<SP24_F16, SP24_F32>(a, experts, st) : run_segments<SP24_F16, SP24_F16>(a, experts, st);
    return a.out == SP24_F32 ? run_segments<SP24_BF16, SP24_F32>(a, experts, st) : run_segments<SP24_BF16, SP24_BF16>(a, experts, st);
}

} // namespace sp24
