// The weights' gradient from few tokens' rows, one operand in 8 bits: D = A^T B as gemm_tokens.hpp has it, B made from codes and scales on its way to LDS.
//
// What a product of a few steps of K costs is launches, the first loads' latency and its result's stores: restored rows would be one launch more.  Codes
// and scales of the next step are on their way in registers while this one is multiplied, and become 16-bit values behind it; every tile of rows converts them
// again, which longer products cannot afford (4096 x 1024 from 8192 tokens, with stages and wavefronts of its own for it: 97 us against 78 for restoring and product).
// 4096 x 1024 bf16 from 64 tokens 5.3 us in a graph, restoring and product 8.0; 8192 x 4096 20.3, 67 MB of results at 3.3 TB/s.
#include "gemm_tokens.hpp"
#include "kept.hpp"

namespace sp24 {

// The rows of a segment (or all) and what the rows of B are made of
struct CodeArgs : TokenArgs {
    const void* codes;
    const float* scale;
    const int32_t* rows;                  // null: row k of the codes
    int64_t tokens, ldc;
    int topk;

    // this workgroup's rows: A from there on, `first` the number of the first
    __device__ __forceinline__ int64_t enter_segment()
    {
        if (!offsets) return 0;
        const int e = blockIdx.y;
        int64_t first, last;
        segment_of(offsets, e, K, first, last);
        A = reinterpret_cast<const uint8_t*>(A) + first * lda * esize_of(in);
        D = reinterpret_cast<uint8_t*>(D) + e * M * ldd * esize_of(out);
        K = last - first;
        return first;
    }
};

template <int DT, int CODE, int OUT, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_codes(CodeArgs a, int tiles_m, int tiles_n)
{
    constexpr int NW = WM * WN, BM = 32 * TM * WM, BN = 32 * TN * WN, BK = kRowBytes / 2;
    using deal_a = deal<BM / 8, NW>;
    using deal_b = deal<BN / 8, NW>;
    constexpr int NJA = deal_a::each, NJB = deal_b::each;
    constexpr int kStageBytes = (BM + BN) * kRowBytes, kEpiBytes = NW * store_bytes<CodeArgs, OUT, TM, TN>();
    __shared__ __attribute__((aligned(1024))) uint8_t lds_all[2 * kStageBytes > kEpiBytes ? 2 * kStageBytes : kEpiBytes];
    int tm, tn;
    tile_of_workgroup(tiles_m, tiles_n, tm, tn);
    const int64_t first = a.enter_segment();
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const int length = (int)a.K, steps = (length + BK - 1) / BK;

    const int64_t lda_bytes = a.lda * 2;
    const uint8_t* const a_blk = reinterpret_cast<const uint8_t*>(a.A) + (int64_t)tm * BM * 2;
    uint32_t a_off[NJA];
    dma_offsets_nmajor<BM, NW, 2>((int64_t)tm * BM, (a.M + 7) / 8 * 8, lda_bytes, wave, lane, a_off);
    nmajor_frags<BM, TM, 2> a_nm;
    nmajor_frags<BN, TN, 2> b_nm;
    a_nm.init(wm, lane);
    b_nm.init(wn, lane);

    // Piece j of a step: eight columns of one of its rows, where the transfers of a 16-bit B would put them
    const int64_t blocks = kept_blocks(a.N);
    int row[NJB], have[NJB];
    const uint8_t* codes[NJB];
    const float* scale[NJB];
#pragma unroll
    for (int j = 0; j < NJB; ++j) {
        const int p = deal_b::id(wave, j) * 1024 + lane * 16;
        row[j] = p / (BN * 2);
        const int64_t at = (int64_t)tn * BN + ((((p % (BN * 2)) >> 4) ^ nmajor_swizzle<2>(row[j], BN / 8)) * 8), col = min(at, a.N - 1);
        have[j] = (int)min(a.N - col, (int64_t)8);               // (columns behind the last are made of its code, and not stored)
        codes[j] = reinterpret_cast<const uint8_t*>(a.codes) + col;
        scale[j] = a.scale + col / kKeptBlock;
    }
    uint2v q[NJB];
    float s[NJB];
    bool live[NJB];
    auto load = [&](int step) {
#pragma unroll
        for (int j = 0; j < NJB; ++j) {
            const int k = step * BK + row[j];
            live[j] = k < length;
            int64_t n = first + min(k, length - 1);
            if (a.rows) {
                const int choice = a.rows[n];
                const uint32_t token = (uint32_t)choice / (uint32_t)a.topk;
                live[j] = live[j] && choice >= 0 && (int64_t)token < a.tokens;
                n = live[j] ? (int64_t)token : 0;
            }
            q[j] = load_codes8<false>(codes[j] + n * a.ldc, have[j]);
            s[j] = scale[j][n * blocks];
        }
    };
    auto put = [&](uint8_t* stage) {
#pragma unroll
        for (int j = 0; j < NJB; ++j) {
            float v[8];
            kept_values8<CODE>(q[j], s[j], v);
            uint4v w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = live[j] ? pack_out16<DT>(v[2 * i], v[2 * i + 1]) : 0u;
            *reinterpret_cast<uint4v*>(stage + BM * kRowBytes + deal_b::id(wave, j) * 1024 + lane * 16) = w;
        }
    };
    auto transfer = [&](int step, uint8_t* stage) {
        const int left = (length - step * BK) * 2;               // bytes of a column of A; rows behind the last are zeros
#pragma unroll
        for (int j = 0; j < NJA; ++j)
            lds_dma_tail<false>(a_blk + step * (BK * lda_bytes), a_off[j], past_k_nmajor<BM, NW, 2>(j, wave, lane, left), stage + deal_a::id(wave, j) * 1024);
    };
    auto all_there = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0) & ~(15 << 8));
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    float16v acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = float16v{};
    if (steps > 0) {
        load(0);
        transfer(0, lds_all);
        put(lds_all);
        all_there();
        for (int step = 0; step < steps; ++step) {
            const uint8_t* const stage = lds_all + (step & 1) * kStageBytes;
            uint8_t* const next = lds_all + (~step & 1) * kStageBytes;      // last read a step ago, in front of the barrier
            const bool more = step + 1 < steps;
            if (more) {
                load(step + 1);
                transfer(step + 1, next);
            }
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                int4v xa[TM], xb[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) xa[i] = __builtin_bit_cast(int4v, a_nm.piece(stage, jj, i));
#pragma unroll
                for (int j = 0; j < TN; ++j) xb[j] = __builtin_bit_cast(int4v, b_nm.piece(stage + BM * kRowBytes, jj, j));
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[i][j] = mfma32<DT>(xa[i], xb[j], acc[i][j]);
            }
            if (more) put(next);
            all_there();
        }
    }
    uint8_t* const scratch = lds_all + wave * store_bytes<CodeArgs, OUT, TM, TN>();
    store_wave_tile<DT, OUT, TM, TN>(a, acc, scratch, (int64_t)tm * BM + wm * TM * 32, (int64_t)tn * BN + wn * TN * 32, lane);
}

template <int DT, int CODE, int OUT>
static sp24_status gemm_codes(const CodeArgs& a, int experts, hipStream_t st)
{
    auto run = [&](auto kernel, int tile, int threads) {
        const int64_t tiles_m = (a.M + tile - 1) / tile, tiles_n = (a.N + tile - 1) / tile;
        return launch_tiles(tiles_m * tiles_n, experts, threads, [&](dim3 grid, dim3 block) { kernel<<<grid, block, 0, st>>>(a, (int)tiles_m, (int)tiles_n); });
    };
    // Small tiles while the chip has room: 1024 x 1000 from 64 tokens on 64 x 64 4.3 us, 128 x 128 5.0; 4096 x 1024 5.7 and 5.3, 8192 x 4096 25.9 and 20.3.
    if ((a.M + 63) / 64 * ((a.N + 63) / 64) * experts <= 512) return run(k_gemm_codes<DT, CODE, OUT, 2, 2, 1, 1>, 64, 256);
    return run(k_gemm_codes<DT, CODE, OUT, 2, 4, 2, 1>, 128, 512);
}

sp24_status launch_gemm_codes(const TokenArgs& t, const RestoreArgs& r, int experts, hipStream_t st)
{
    CodeArgs a{};
    static_cast<TokenArgs&>(a) = t;
    a.codes = r.codes;
    a.scale = r.scale;
    a.rows = r.rows;
    a.tokens = r.N;
    a.ldc = r.ldc;
    a.topk = r.topk;
    auto by_code = [&](auto dt, auto out) {
        constexpr int DT = decltype(dt)::value, OUT = decltype(out)::value;
        return r.code == SP24_I8 ? gemm_codes<DT, SP24_I8, OUT>(a, experts, st) : gemm_codes<DT, SP24_F8, OUT>(a, experts, st);
    };
    const std::integral_constant<int, SP24_F16> f16;
    const std::integral_constant<int, SP24_BF16> bf16;
    const std::integral_constant<int, SP24_F32> f32;
    if (t.in == SP24_F16) return t.out == SP24_F32 ? by_code(f16, f32) : by_code(f16, f16);
    return t.out == SP24_F32 ? by_code(bf16, f32) : by_code(bf16, bf16);
}

} // namespace sp24
