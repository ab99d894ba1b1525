// The weights' gradient from rows kept in 8 bits: D = A B, A the transposed gradient of a layer's result (M x tokens, 16 bits), B what codes and
// scales stand for (tokens x N), for all tokens or for every expert's.
//
// A goes to LDS by transfers, as in the product of two 16-bit matrices; B comes through registers, where codes become 16-bit values, and
// lies in LDS as rows of tokens, from which the transposing reads take the fragments.
#include "kept.hpp"
#include "linear.hpp"
#include "mm_tiled.hpp"

namespace sp24 {

template <int DT, int CODE, int OUT, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN, 1) void k_gemm_kept(KeptMmArgs g, int tiles_m, int tiles_n)
{
    constexpr int NW = WM * WN, BM = 32 * TM * WM, BN = 32 * TN * WN, BK = kRowBytes / 2;
    constexpr int kRowB = BN * 2, kChunks = kRowB / 16, kPieces = BN / 16;                  // of a token's row in LDS; pieces of 16 codes
    constexpr int NB = BK * kPieces / (64 * NW);
    constexpr int kStageBytes = BM * kRowBytes + BK * kRowB;
    constexpr int kEpiBytes = NW * epilogue_geometry<OUT, TN>::kWaveBytes;
    static_assert(BK * kPieces % (64 * NW) == 0, "the threads share a step's codes evenly");
    __shared__ __attribute__((aligned(1024))) uint8_t lds_all[kStageBytes > kEpiBytes ? kStageBytes : kEpiBytes];
    uint8_t* const lds_b = lds_all + BM * kRowBytes;

    int tm, tn;
    tile_of_workgroup(tiles_m, tiles_n, tm, tn);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, r = lane & 31, q = lane >> 5;
    int64_t first = 0, last = g.K;
    if (g.offsets) segment_of(g.offsets, blockIdx.y, g.K, first, last);
    const int64_t K = last - first;
    const int nsteps = (int)(K / BK), tail = (int)(K % BK) * 2;                             // whole steps; bytes of K in one more

    const int64_t lda_bytes = g.lda * 2;
    const uint8_t* const a_blk = reinterpret_cast<const uint8_t*>(g.A) + (int64_t)tm * BM * lda_bytes + first * 2;
    uint32_t a_off[deal<BM / 8, NW>::each];
    dma_offsets<BM, NW>((int64_t)tm * BM, g.M, lda_bytes, wave, lane, a_off);
    int fa_off[4];
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) fa_off[jj] = (wm * 32 * TM + r) * kRowBytes + ((((2 * jj) | q) ^ ((r >> 1) & 7)) << 4);
    nmajor_frags<BN, TN, 2> b_nm;
    b_nm.init(wn, lane);

    const int64_t blocks = (g.N + kKeptBlock - 1) / kKeptBlock;
    // piece x of this thread: 16 codes of one token's row
    auto fetch = [&](int step, int x, uint4v& codes, float& scale) {
        const int p = tid + x * 64 * NW, row = p / kPieces, c = p % kPieces;
        const int64_t k = first + (int64_t)step * BK + row, col = (int64_t)tn * BN + c * 16;
        codes = uint4v{0, 0, 0, 0};
        scale = 0.0f;
        if (k >= last || col >= g.N) return;
        int64_t token = k;
        if (g.rows) {
            const int choice = g.rows[k];
            token = choice < 0 ? -1 : choice / g.topk;
        }
        if (token < 0 || token >= g.tokens) return;
        const uint8_t* const at = reinterpret_cast<const uint8_t*>(g.codes) + token * g.ldc + col;
        scale = g.scale[token * blocks + col / kKeptBlock];
        if (col + 16 <= g.N) codes = load_from<uint4v>(at);
        else {
            const int have = (int)(g.N - col);
            for (int i = 0; i < 16; ++i)
                if (i < have) codes[i / 4] |= (uint32_t)at[i] << (8 * (i % 4));
        }
    };
    auto put = [&](int x, const uint4v& codes, float scale) {
        const int p = tid + x * 64 * NW, row = p / kPieces, c = p % kPieces;
        uint4v v[2];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            float f[4];
            code_values4<CODE>(codes[d], f);
            v[d / 2][2 * (d % 2)] = pack_out16<DT>(f[0] * scale, f[1] * scale);
            v[d / 2][2 * (d % 2) + 1] = pack_out16<DT>(f[2] * scale, f[3] * scale);
        }
        uint8_t* const to = lds_b + row * kRowB + (((2 * c) ^ nmajor_swizzle<2>(row, kChunks)) << 4);
        *reinterpret_cast<uint4v*>(to) = v[0];
        *reinterpret_cast<uint4v*>(to + 16) = v[1];
    };

    float16v acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = float16v{};
    for (int step = 0; step < nsteps + (tail != 0); ++step) {
        const bool partial = step == nsteps;
#pragma unroll
        for (int j = 0; j < deal<BM / 8, NW>::each; ++j) {
            uint8_t* const to = lds_all + deal<BM / 8, NW>::id(wave, j) * 1024;
            if (partial) lds_dma_tail<false>(a_blk + (int64_t)step * kRowBytes, a_off[j], past_k_kmajor<BM, NW>(j, wave, lane, tail), to);
            else lds_dma16(a_blk + (int64_t)step * kRowBytes, a_off[j], to);
        }
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            uint4v codes;
            float scale;
            fetch(step, x, codes, scale);
            put(x, codes, scale);
        }
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __syncthreads();
        if (partial && tail % 16 != 0) {
            // K ends inside a 16-byte piece of A's rows: what lies there behind K is not the matrix's, and a NaN would outlast B's zeros
            for (int row = tid; row < BM; row += 64 * NW) {
                uint16_t* const piece = reinterpret_cast<uint16_t*>(lds_all + row * kRowBytes + (((tail >> 4) ^ ((row >> 1) & 7)) << 4));
                for (int i = tail % 16 / 2; i < 8; ++i) piece[i] = 0;
            }
            __syncthreads();
        }
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
            int4v fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = *reinterpret_cast<const int4v*>(lds_all + fa_off[jj] + i * 32 * kRowBytes);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = __builtin_bit_cast(int4v, b_nm.piece(lds_b, jj, j));
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[i][j] = mfma32<DT>(fa[i], fb[j], acc[i][j]);
        }
        __syncthreads();
    }
    MmArgs a{};
    a.D = reinterpret_cast<uint8_t*>(g.D) + (int64_t)blockIdx.y * g.M * g.ldd * out_size<OUT>();
    a.M = g.M;
    a.N = g.N;
    a.ldd = g.ldd;
    store_wave_tile<DT, OUT, TM, TN>(a, acc, lds_all + wave * epilogue_geometry<OUT, TN>::kWaveBytes, (int64_t)tm * BM + wm * TM * 32,
                                     (int64_t)tn * BN + wn * TN * 32, lane);
}

template <int DT, int CODE, int OUT>
static sp24_status run_kept(const KeptMmArgs& a, hipStream_t st)
{
    const int64_t tiles_m = (a.M + 127) / 128, tiles_n = (a.N + 127) / 128;
    return launch_tiles(tiles_m * tiles_n, a.experts, 256, [&](dim3 grid, dim3 block) {
        k_gemm_kept<DT, CODE, OUT, 2, 2, 2, 2><<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n);
    });
}

template <int DT, int CODE>
static sp24_status by_output(const KeptMmArgs& a, hipStream_t st)
{
    return a.out == SP24_F32 ? run_kept<DT, CODE, SP24_F32>(a, st) : run_kept<DT, CODE, DT>(a, st);
}

sp24_status launch_gemm_kept(const KeptMmArgs& a, hipStream_t st)
{
    if (a.in == SP24_F16) return a.code == SP24_I8 ? by_output<SP24_F16, SP24_I8>(a, st) : by_output<SP24_F16, SP24_F8>(a, st);
    return a.code == SP24_I8 ? by_output<SP24_BF16, SP24_I8>(a, st) : by_output<SP24_BF16, SP24_F8>(a, st);
}

} // namespace sp24
