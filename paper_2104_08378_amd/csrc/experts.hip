// Tokens in order of their expert and back: the sort of the router's choices, the rows gathered, the weighted sum of what comes back, and
// that sum's gradients.
#include <algorithm>

#include "launch.hpp"
#include "rowops.hpp"

namespace sp24 {

// ---------------------------------------------------------------------------
// The sort is a counting sort that keeps the order of equal keys: how many choices every expert has in all and before a wavefront's 64, and
// the place of each among the 64 (ballots over the bits of the expert's number).  Whole numbers throughout, so the result is one.
//
// Placing takes some 85 instructions to 64 choices, which one compute unit issues at 0.5 us a thousand (4096 x 2 choices of eight 8.7 us on one
// workgroup), counting a few: every workgroup counts all choices, from the L2, and places a thousand, one launch and nothing to wait for (5.7 us; 4096 x 4
// of 64 16.7 -> 6.2).
// Past kSortAtOnce choices parts of kSortPart count, a scan over parts and experts, and parts place: three launches whose time hardly grows, where
// counting everything in every workgroup grows with the square.  One launch / parts, us, uniform choices: of 8 experts 2^13 6.1 / 15.1, 2^16
// 18.1 / 21.3, 2^17 32 / 21.3, 2^18 60 / 22.4, 2^20 800 / 28; of 64 2^13 5.6 / 17.8, 2^16 12.4 / 27.2, 2^17 20.4 / 27.2, 2^18 38 / 28.4; of 1024 2^13 9.9 /
// 27.4, 2^17 25.1 / 42.4, 2^18 44.1 / 43.6.  2^17 is between the experts' numbers: right for 64, past the crossing for 8 (about 2^16), before it for 1024.
// ---------------------------------------------------------------------------
constexpr int kSortWaves = 16, kSortExperts = 1024;

struct SortLds {
    int count[kSortWaves][kSortExperts];       // of a wavefront's part; then the next row it gives out
    int scan[kSortWaves];
};

// lanes with the same key as this one, among those with `live`
template <int BITS>
__device__ __forceinline__ uint64_t same_key(int key, bool live)
{
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const uint64_t set = __ballot((key >> b) & 1);
        same &= (key >> b) & 1 ? set : ~set;
    }
    return same;
}

// A lane's RUNS choices: the expert, or -1, and how many of the wavefront's earlier ones name the same.
template <int RUNS>
struct SortRun {
    int expert[RUNS], before[RUNS];
};

// The wavefront's n choices from `ids` on, at most 64 RUNS: leaves in count[] how many of them each expert has.
template <int BITS, int RUNS>
__device__ __forceinline__ void sort_count(int* count, const int32_t* ids, int n, int experts, SortRun<RUNS>& run)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int u = 0; u < RUNS; ++u) run.expert[u] = u * 64 + lane < n ? ids[u * 64 + lane] : -1;
    for (int e = lane; e < experts; e += 64) count[e] = 0;
#pragma unroll
    for (int u = 0; u < RUNS; ++u) {
        if (u * 64 >= n) continue;
        const int e = run.expert[u];
        const bool live = (unsigned)e < (unsigned)experts;
        const uint64_t same = same_key<BITS>(e, live);
        if (!live) {
            run.expert[u] = -1;
            continue;
        }
        const int before = count[e];
        run.before[u] = before + __popcll(same & (((uint64_t)1 << lane) - 1));
        if (__ffsll((unsigned long long)same) - 1 == lane) count[e] = before + __popcll(same);
    }
}

// Their rows, count[] holding the first row that the wavefront has of each expert; `number` is that of the first choice.
template <int RUNS>
__device__ __forceinline__ void sort_place(const int* count, const SortArgs& a, const SortRun<RUNS>& run, int64_t number, int n)
{
    const int lane = threadIdx.x & 63;
    int32_t* const slots = a.slots + number;
#pragma unroll
    for (int u = 0; u < RUNS; ++u) {
        const int i = u * 64 + lane;
        if (i >= n) continue;
        int row = -1;
        if (run.expert[u] >= 0) {
            row = count[run.expert[u]] + run.before[u];
            a.rows[row] = (int32_t)number + i;
        }
        slots[i] = row;
    }
}

// Segments from the experts' totals (thread e holds that of expert e): whole sixteens one behind the other.  Returns the segment's first row;
// *end: the end of the last.
__device__ __forceinline__ int sort_segments(int* scan, int total, int* end)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int padded = (total + 15) & ~15;
    int upto = padded;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int t = __shfl_up(upto, d);
        if (lane >= d) upto += t;
    }
    if (lane == 63) scan[wave] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        if (w < wave) before += scan[w];
        all += scan[w];
    }
    *end = all;
    return before + upto - padded;
}

// offsets, and -1 in the rows that no choice has (thread e: those of expert e; all threads: those behind the last segment)
__device__ __forceinline__ void sort_finish(const SortArgs& a, int first, int total, int end)
{
    const int e = threadIdx.x;
    if (e < a.experts) {
        a.offsets[e] = first;
        for (int i = first + total; i < first + ((total + 15) & ~15); ++i) a.rows[i] = -1;
    }
    if (e == 0) a.offsets[a.experts] = end;
    for (int64_t i = end + threadIdx.x; i < a.R; i += blockDim.x) a.rows[i] = -1;
}

// from an expert's first row, thread e: that of every wavefront
__device__ __forceinline__ void sort_first_rows(SortLds& s, int e, int next)
{
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const int n = s.count[w][e];
        s.count[w][e] = next;
        next += n;
    }
}

// All of the sort, workgroup p placing choices 1024 p .. 1024 p + 1023.  (Up to eight experts counted in fields of a register, and those
// added over the wavefront, took 0.9 us longer than the additions in LDS, 64 to eight words though they are.)
template <int BITS>
__global__ __launch_bounds__(1024) void k_sort_at_once(SortArgs a)
{
    __shared__ SortLds s;
    __shared__ int before[kSortExperts], after[kSortExperts];   // choices of each expert in the parts before this one; in the others
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = blockIdx.x, T = (int)a.T, parts = (T + 1023) / 1024;
    if (parts > 1) {                                            // (else the wavefronts' counts below say it all)
        before[tid] = after[tid] = 0;
        __syncthreads();
        for (int p0 = 0; p0 < parts; p0 += 8) {                  // eight loads on their way
            int expert[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = (p0 + u) * 1024 + tid;
                expert[u] = i < T ? a.ids[i] : -1;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int e = expert[u];
                const bool live = (unsigned)e < (unsigned)a.experts, earlier = p0 + u < part;
                // (a run of one expert is one addition, not 64 to one word)
                int* const sum = earlier ? before : after;
                if (__ballot(e == __builtin_amdgcn_readfirstlane(e)) == ~(uint64_t)0) {
                    if (lane == 0 && live) atomicAdd(&sum[e], 64);
                } else if (live) atomicAdd(&sum[e], 1);
            }
        }
    }
    const int number = part * 1024 + wave * 64, n = min(max(T - number, 0), 64);
    SortRun<1> run;
    sort_count<BITS>(s.count[wave], a.ids + number, n, a.experts, run);
    __syncthreads();
    int mine = 0, total = 0;
    if (tid < a.experts && parts > 1) {
        mine = before[tid];
        total = mine + after[tid];
    } else if (tid < a.experts) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) total += s.count[w][tid];
    }
    int end;
    const int first = sort_segments(s.scan, total, &end);
    if (tid < a.experts) sort_first_rows(s, tid, first + mine);
    if (part == 0) sort_finish(a, first, total, end);
    __syncthreads();
    sort_place(s.count[wave], a, run, number, n);
}

constexpr int kSortRuns = kSortPart / kSortWaves / 64;          // of 64 choices, to a wavefront of a part

// a wavefront's choices of part blockIdx.x: equal runs of whole 64s
__device__ __forceinline__ void sort_share(const SortArgs& a, int64_t& number, int& n)
{
    const int64_t first = (int64_t)blockIdx.x * kSortPart;
    const int in_part = (int)min((int64_t)kSortPart, a.T - first), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    number = first + wave * 64 * kSortRuns;
    n = min(max(in_part - wave * 64 * kSortRuns, 0), 64 * kSortRuns);
}

template <int BITS>
__global__ __launch_bounds__(1024) void k_sort_count(SortArgs a)
{
    __shared__ SortLds s;
    SortRun<kSortRuns> run;
    int64_t number;
    int n;
    sort_share(a, number, n);
    sort_count<BITS>(s.count[threadIdx.x >> 6], a.ids + number, n, a.experts, run);
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) {
        int total = 0;
        for (int w = 0; w < kSortWaves; ++w) total += s.count[w][e];
        a.workspace[(int64_t)blockIdx.x * a.experts + e] = total;
    }
}

// counts of the parts -> the first row that each part gives out
__global__ __launch_bounds__(1024) void k_sort_scan(SortArgs a, int parts)
{
    __shared__ int scan[kSortWaves];
    const int e = threadIdx.x;
    int total = 0;
    if (e < a.experts) {
#pragma unroll 8
        for (int p = 0; p < parts; ++p) total += a.workspace[(int64_t)p * a.experts + e];
    }
    int end;
    const int first = sort_segments(scan, total, &end);
    if (e < a.experts) {
        int next = first;
#pragma unroll 8
        for (int p = 0; p < parts; ++p) {
            const int n = a.workspace[(int64_t)p * a.experts + e];
            a.workspace[(int64_t)p * a.experts + e] = next;
            next += n;
        }
    }
    sort_finish(a, first, total, end);
}

template <int BITS>
__global__ __launch_bounds__(1024) void k_sort_place(SortArgs a)
{
    __shared__ SortLds s;
    SortRun<kSortRuns> run;
    int64_t number;
    int n;
    sort_share(a, number, n);
    sort_count<BITS>(s.count[threadIdx.x >> 6], a.ids + number, n, a.experts, run);
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) sort_first_rows(s, e, a.workspace[(int64_t)blockIdx.x * a.experts + e]);
    __syncthreads();
    sort_place(s.count[threadIdx.x >> 6], a, run, number, n);
}

template <int BITS>
static void run_sort(const SortArgs& a, hipStream_t st)
{
    if (a.T <= kSortAtOnce) {
        const unsigned parts = a.T > 1024 ? (unsigned)((a.T + 1023) / 1024) : 1u;
        k_sort_at_once<BITS><<<parts, 1024, 0, st>>>(a);
        return;
    }
    const int parts = (int)((a.T + kSortPart - 1) / kSortPart);
    k_sort_count<BITS><<<parts, 1024, 0, st>>>(a);
    k_sort_scan<<<1, 1024, 0, st>>>(a, parts);
    k_sort_place<BITS><<<parts, 1024, 0, st>>>(a);
}

sp24_status launch_moe_sort(const SortArgs& a, hipStream_t st)
{
    if (a.experts <= 8) run_sort<3>(a, st);
    else if (a.experts <= 64) run_sort<6>(a, st);
    else run_sort<10>(a, st);
    return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
}

// ---------------------------------------------------------------------------
// Rows by expert: row i is the token of choice rows[i], zeros where there is none.  Bound by memory, 16 bytes a thread.
// 4096 tokens of 4096 bf16 to two experts each: 21.2 us, 101 MB at 4.7 TB/s where a token is counted once; int8 with scales 12.1 (4.2), 16 tokens 2.6.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint4v load_bytes(const uint8_t* p, int64_t n)
{
    if (n >= 16) return load_from<uint4v>(p);
    uint4v v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) v[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    return v;
}
__device__ __forceinline__ void store_bytes(uint8_t* p, int64_t n, const uint4v& v)
{
    if (n >= 16) {
        store_to(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) p[i] = (uint8_t)(v[i / 4] >> (8 * (i % 4)));
}

__global__ __launch_bounds__(256) void k_moe_gather(GatherArgs a, int blocks_a_row, unsigned from)
{
    const unsigned group = from + blockIdx.x;
    const int64_t row = group / blocks_a_row;
    const int64_t at = ((int64_t)(group % blocks_a_row) * blockDim.x + threadIdx.x) * 16;
    const int64_t choice = a.rows[row], token = choice < 0 ? -1 : choice / a.topk;
    const bool live = token >= 0 && token < a.N;
    if (a.scale_out && at == 0) a.scale_out[row] = live ? a.scale[token] : 0.0f;
    if (at >= a.row_bytes) return;
    const int64_t n = a.row_bytes - at;
    const uint4v v = live ? load_bytes(reinterpret_cast<const uint8_t*>(a.X) + token * a.ldx_bytes + at, n) : uint4v{0u, 0u, 0u, 0u};
    store_bytes(reinterpret_cast<uint8_t*>(a.Xs) + row * a.ldxs_bytes + at, n, v);
}

// a launch of threads that hold `width` bytes (values) of a row each: threads of a workgroup, workgroups to a row
static void row_launch(int64_t length, int width, unsigned& threads, int& blocks_a_row)
{
    const int64_t pieces = (length + width - 1) / width;
    threads = (unsigned)(pieces >= 256 ? 256 : (pieces + 63) / 64 * 64);
    blocks_a_row = (int)((pieces + threads - 1) / threads);
}

sp24_status launch_moe_gather(const GatherArgs& a, hipStream_t st)
{
    unsigned threads;
    int blocks;
    row_launch(a.row_bytes, 16, threads, blocks);
    return launch_in_parts(a.R * blocks, threads, [&](unsigned from, unsigned grid) { k_moe_gather<<<grid, threads, 0, st>>>(a, blocks, from); });
}

// ---------------------------------------------------------------------------
// out[n] = residual[n] + sum over j, in that order, of weights[n][j] Y[slots[n][j]], in binary32, rounded once.  Bound by memory, eight
// values a thread.  4096 tokens of 4096 bf16 from two experts each, with residual: 22.0 us, 134 MB at 6.1 TB/s.  (Y, residual and out have one type:
// the experts' results come rounded to it, and out is; a float32 stream takes float32 results.)
// ---------------------------------------------------------------------------
template <int T>
__global__ __launch_bounds__(256) void k_moe_combine(CombineArgs a, int blocks_a_row, unsigned from)
{
    const unsigned group = from + blockIdx.x;
    const int64_t n = group / blocks_a_row;
    const int64_t at = ((int64_t)(group % blocks_a_row) * blockDim.x + threadIdx.x) * 8;
    if (at >= a.H) return;
    const int have = (int)min(a.H - at, (int64_t)8);
    float sum[8] = {};
    raw8<T> first = {};
    if (a.residual) first = load_raw8<T>(a.residual, n * a.ldr + at, have);
    for (int j0 = 0; j0 < a.topk; j0 += 4) {                     // four rows on their way
        raw8<T> y[4];
        float w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u;
            const int64_t slot = j < a.topk ? a.slots[n * a.topk + j] : -1;
            const bool live = slot >= 0 && slot < a.R;
            w[u] = !live ? 0.0f : a.weights ? a.weights[n * a.topk + j] : 1.0f;
            y[u] = live ? load_raw8<T>(a.Y, slot * a.ldy + at, have) : raw8<T>{};
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float v[8];
            values_of<T>(y[u], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(w[u], v[i], sum[i]);
        }
    }
    if (a.residual) {
        float v[8];
        values_of<T>(first, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
    }
    store_values8<T>(a.out, n * a.ldo + at, have, sum);
}

sp24_status launch_moe_combine(const CombineArgs& a, hipStream_t st)
{
    unsigned threads;
    int blocks;
    row_launch(a.H, 8, threads, blocks);
    return launch_in_parts(a.N * blocks, threads, [&](unsigned from, unsigned grid) {
        if (a.t == SP24_F32) k_moe_combine<SP24_F32><<<grid, threads, 0, st>>>(a, blocks, from);
        else if (a.t == SP24_F16) k_moe_combine<SP24_F16><<<grid, threads, 0, st>>>(a, blocks, from);
        else k_moe_combine<SP24_BF16><<<grid, threads, 0, st>>>(a, blocks, from);
    });
}

// ---------------------------------------------------------------------------
// Its gradients: dY[i] = weight of choice rows[i] times dOut of its token (zeros where there is none), dweights = the inner product of
// dOut and Y there, 0 for a choice without a row.  Bound by memory, a wavefront to a row: both gradients from one read of it.  4096 tokens of
// 1024 bf16 on four experts each, one choice in 20 without a row: 17.6 us, 72 MB at 4.1 TB/s.
// ---------------------------------------------------------------------------
template <int T>
__global__ __launch_bounds__(256) void k_moe_combine_grad(CombineGradArgs a, unsigned from)
{
    const int lane = threadIdx.x & 63;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < a.N * a.topk; t += (int64_t)gridDim.x * 256)      // (in each part again)
        if (a.slots[t] < 0 || a.slots[t] >= a.R) a.dweights[t] = 0.0f;
    const int64_t row = ((int64_t)from + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= a.R) return;
    const int64_t choice = a.rows[row], token = choice < 0 ? -1 : choice / a.topk;
    const bool live = token >= 0 && token < a.N;
    const float w = live ? a.weights[choice] : 0.0f;
    float dot = 0.0f;
    for (int64_t at = lane * 8; at < a.H; at += 512) {
        const int have = (int)min(a.H - at, (int64_t)8);
        float d[8] = {}, y[8];
        if (live) {
            values_of<T>(load_raw8<T>(a.dOut, token * a.lddo + at, have), d);
            values_of<T>(load_raw8<T>(a.Y, row * a.ldy + at, have), y);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dot = __builtin_fmaf(d[i], y[i], dot);
                d[i] *= w;
            }
        }
        store_values8<T>(a.dY, row * a.lddy + at, have, d);
    }
    dot = __uint_as_float(over_wave<add_f>(__float_as_uint(dot)));
    if (live && lane == 0) a.dweights[choice] = dot;
}

sp24_status launch_moe_combine_grad(const CombineGradArgs& a, hipStream_t st)
{
    const int64_t groups = std::max<int64_t>((a.R + 3) / 4, 1);                // (choices without rows have gradients to write)
    return launch_in_parts(groups, 256, [&](unsigned from, unsigned grid) {
        if (a.t == SP24_F32) k_moe_combine_grad<SP24_F32><<<grid, 256, 0, st>>>(a, from);
        else if (a.t == SP24_F16) k_moe_combine_grad<SP24_F16><<<grid, 256, 0, st>>>(a, from);
        else k_moe_combine_grad<SP24_BF16><<<grid, 256, 0, st>>>(a, from);
    });
}

} // namespace sp24
