// The experts of every token from the router's logits, and the gradient of what comes of it.
//
//   s = softmax(l) or 1 / (1 + e^-l),  c = s + bias;  the experts of the largest c, their weights s / sum s (or s) times scale
//   g[e] = ds[e] + sum over j of [ids[j] = e] dg[j],  dg = scale (dw - sum(dw s) / W) / W  (not renormalised: scale dw),  W = sum of the chosen s
//   softmax: dl = s (g - sum g s);  logistic: dl = s (1 - s) g
//
// All in binary64: of 10^5 tokens' experts some pairs' scores are within a rounding of binary32 of each other, and which one is chosen must
// not hang on how the sum was taken; within one of binary64 the sum's order decides, which is the same whatever the number of rows.
//
// Bound by vector operations, two thirds of the time busy with them: an exponential of some 35 in binary64 for every logit, and for every choice the
// reduction over the row's lanes and a search in the one that has it.  Few rows: a launch and one row's chain of them.  In a graph, us: 16 rows, four of 64 experts
// 2.9; 8192 rows, six of 64 4.5, eight of 256 9.8, by logistic scores with bias out of four of eight groups 10.6 (1.4 is what their 8.9 MB take), six of 160
// out of three of eight groups, which are no run of whole lanes, 13.3; 2048 rows of 1024 10.0; the gradient of 8192 rows of 256 with that of the scores 9.0 (25 MB: 4.1).  (An exponential
// for arguments below 0 alone, of 25 operations in place of 37, changed none of it.)
#include <algorithm>

#include "launch.hpp"
#include "rowops.hpp"

namespace sp24 {

constexpr int kRouteThreads = 256;

// ---- L lanes (a power of two) hold a row, lane l its experts l * V .. l * V + V - 1, so that the lowest lane has the lowest experts ----

template <int CTRL>
__device__ __forceinline__ double dpp_of(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// OP of both sixteens of every 32 lanes, or (WAVE) of both halves of the wavefront, in all of them: a register swapped with a copy of itself leaves the
// lower one in both places of the one and the upper one in both of the other
template <bool WAVE, class OP>
__device__ __forceinline__ double over_halves(double v, OP op)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)b, hi = (uint32_t)(b >> 32);
    auto swapped = [](uint32_t x) {
        if constexpr (WAVE) return __builtin_amdgcn_permlane32_swap(x, x, false, false);
        else return __builtin_amdgcn_permlane16_swap(x, x, false, false);
    };
    const auto l = swapped(lo), h = swapped(hi);
    return op(__builtin_bit_cast(double, ((uint64_t)h[0] << 32) | l[0]), __builtin_bit_cast(double, ((uint64_t)h[1] << 32) | l[1]));
}
// OP over the L lanes of a row, the same in all of them and in the same order always
template <int L, class OP>
__device__ __forceinline__ double over_row(double v, OP op)
{
    if constexpr (L >= 2) v = op(v, dpp_of<0xB1>(v));            // quad_perm [1,0,3,2]
    if constexpr (L >= 4) v = op(v, dpp_of<0x4E>(v));            // quad_perm [2,3,0,1]
    if constexpr (L >= 8) v = op(v, dpp_of<0x141>(v));           // the other half of eight lanes, mirrored
    if constexpr (L >= 16) v = op(v, dpp_of<0x140>(v));          // the other half of sixteen
    if constexpr (L >= 32) v = over_halves<false>(v, op);
    if constexpr (L >= 64) v = over_halves<true>(v, op);
    return v;
}
struct larger_of { __device__ __forceinline__ double operator()(double a, double b) const { return __builtin_fmax(a, b); } };
struct sum_of {
    __device__ __forceinline__ double operator()(double a, double b) const
    {
#pragma clang fp contract(off)
        return a + b;                                            // (a product that is added is rounded first, wherever it stands)
    }
};
// The sum over a row, neighbouring experts first, then neighbouring pairs and so on, so that it does not hang on how many lanes share the row's experts,
// which goes by the number of rows: a row's choice would (as fast as a lane's values one after the other).
template <int COUNT>
__device__ __forceinline__ double sum_of_neighbours(const double (&v)[COUNT])
{
    double part[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) part[i] = v[i];
#pragma unroll
    for (int d = 1; d < COUNT; d *= 2)
#pragma unroll
        for (int i = 0; i < COUNT; i += 2 * d) part[i] = sum_of{}(part[i], part[i + d]);
    return part[0];
}
template <int L, int V>
__device__ __forceinline__ double sum_of_row(const double (&v)[V])
{
    return over_row<L>(sum_of_neighbours(v), sum_of{});
}
// The same of a row's `topk` choices, lane l with choices l, L + l, ...: a run of L choices in every part
template <int L, int PARTS>
__device__ __forceinline__ double sum_of_choices(const double (&v)[PARTS], int topk)
{
    double part[PARTS];
#pragma unroll
    for (int i = 0; i < PARTS; ++i) part[i] = i == 0 || i * L < topk ? over_row<L>(v[i], sum_of{}) : 0.0;
    return sum_of_neighbours(part);
}
template <int L>
__device__ __forceinline__ uint32_t most_of_row(uint32_t v)
{
    if constexpr (L >= 2) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    if constexpr (L >= 4) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
    if constexpr (L >= 8) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
    if constexpr (L >= 16) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
    if constexpr (L >= 32) {
        const auto h = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(h[0], h[1]);
    }
    if constexpr (L >= 64) {
        const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(h[0], h[1]);
    }
    return v;
}
// bits of a number (no NaN) as a whole one of the same order
__device__ __forceinline__ uint32_t in_order(float v)
{
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
// The larger of two that are no NaN: the compiler's own has each quieted first, an operation each.
__device__ __forceinline__ double larger(double a, double b)
{
    double v;
    asm("v_max_f64 %0, %1, %2" : "=v"(v) : "v"(a), "v"(b));
    return v;
}

// COUNT neighbouring values from element i on, the first `have` of them (the others: `otherwise`); 16 bytes at a time where there are that many
template <int T, int COUNT>
__device__ __forceinline__ void load_run(const void* p, int64_t i, int have, float otherwise, float (&v)[COUNT])
{
    constexpr int kAtOnce = T == SP24_F32 ? 4 : 8;
    if (COUNT % kAtOnce == 0 && have >= COUNT) {
        const uint8_t* const at = reinterpret_cast<const uint8_t*>(p) + i * value_size<T>();
#pragma unroll
        for (int k = 0; k < COUNT / kAtOnce; ++k) {
            const uint4v q = load_from<uint4v>(at + k * 16);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if constexpr (T == SP24_F32) v[k * kAtOnce + j] = __uint_as_float(q[j]);
                else v[k * kAtOnce + j] = value_of<T>((q[j / 2] >> (16 * (j & 1))) & 0xFFFFu);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < COUNT; ++k) v[k] = k < have ? load_value<T>(p, i + k) : otherwise;
    }
}
template <int COUNT>
__device__ __forceinline__ void load_logits(const void* p, int64_t i, int have, sp24_dtype t, float (&v)[COUNT])
{
    if (t == SP24_F32) load_run<SP24_F32>(p, i, have, -__builtin_inff(), v);
    else if (t == SP24_BF16) load_run<SP24_BF16>(p, i, have, -__builtin_inff(), v);
    else load_run<SP24_F16>(p, i, have, -__builtin_inff(), v);
}

// COUNT neighbouring results from element i on, the first `have` of them, each rounded to T
template <int T, int COUNT>
__device__ __forceinline__ void store_run(void* p, int64_t i, int have, const float (&v)[COUNT])
{
    constexpr int kAtOnce = T == SP24_F32 ? 4 : 8;
    if (COUNT % kAtOnce == 0 && have >= COUNT) {
        uint8_t* const at = reinterpret_cast<uint8_t*>(p) + i * value_size<T>();
#pragma unroll
        for (int k = 0; k < COUNT / kAtOnce; ++k) {
            uint4v q;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (T == SP24_F32) q[j] = __float_as_uint(v[k * kAtOnce + j]);
                else q[j] = pack_out16<T>(v[k * kAtOnce + 2 * j], v[k * kAtOnce + 2 * j + 1]);
            }
            store_to(at + k * 16, q);
        }
    } else {
#pragma unroll
        for (int k = 0; k < COUNT; ++k)
            if (k < have) store_out<T>(p, i + k, v[k]);
    }
}

constexpr double kNever = -__builtin_inf();
constexpr double kInfinite = 1e300;                              // what +inf is compared as, below a NaN and above all sums of numbers
constexpr uint32_t kChosen = 0xFFEFFFFFu;                        // upper half of -1.8e308

// The scores of a row's experts, 0 for those whose logit is -inf, and (rest) 1 - s of a logistic one without the difference.  A NaN (or, softmax,
// +inf) makes NaN of what it takes part in.  Exponents are 0 and less.
template <int L, int V>
__device__ __forceinline__ void scores_of_row(const float (&x)[V], bool softmax, double (&s)[V], double* rest = nullptr)
{
    if (softmax) {
        float most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < V; ++i) most = fmaxf(most, x[i]);
        const double top = over_row<L>((double)most, larger_of{});
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = x[i] == -__builtin_inff() ? 0.0 : exp((double)x[i] - top);
        const double part = 1.0 / sum_of_row<L>(s);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = x[i] == -__builtin_inff() ? 0.0 : s[i] * part;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            // 1 / (1 + t) for x >= 0 and t / (1 + t) below, t = e^-|x|; the chip's reciprocal with two steps of Newton's: 1 + t is 1 to 2
            const double t = exp(-__builtin_fabs((double)x[i])), d = 1.0 + t;
            double q = __builtin_amdgcn_rcp(d);
            q = __builtin_fma(__builtin_fma(-d, q, 1.0), q, q);
            q = __builtin_fma(__builtin_fma(-d, q, 1.0), q, q);
            s[i] = x[i] < 0.0f ? t * q : q;                      // (0 at -inf)
            if (rest) rest[i] = x[i] < 0.0f ? q : t * q;
        }
    }
}

// lane `from` of the row's L lanes, to all of them
template <int L>
__device__ __forceinline__ double row_lane(double v, int from)
{
    return __shfl(v, from, L);
}

// Where expert e's value lies in a row's image in LDS: first experts of all lanes, then second ones, so that the lanes' writes are neighbours
template <int L, int V>
__device__ __forceinline__ int image_place(int e)
{
    return e % V * L + e / V;
}

// What a group is worth whose largest c are these: their sum, and no more than one that is infinite or NaN
__device__ __forceinline__ double group_value(double first, double second, int best)
{
    return best == 1 || second == kNever || first >= kInfinite ? first : first + second;
}

// How experts are grouped: not; runs of 2^n lanes that hold whole groups; any other way
enum { kNoGroups, kLaneGroups, kAnyGroups };

template <int L, int V, int GROUPS>
__global__ __launch_bounds__(kRouteThreads) void k_route(RouteArgs a, unsigned from)
{
    constexpr int kRows = kRouteThreads / L, kMost = L * V, kPicks = kMost < SP24_MOST_CHOICES ? kMost : SP24_MOST_CHOICES, kParts = (kPicks + L - 1) / L;
    constexpr bool ANY = GROUPS == kAnyGroups;
    __shared__ double scores[kRows][kMost];
    __shared__ int picked[kRows][kPicks];
    __shared__ double keys[ANY ? kRows : 1][ANY ? kMost : 1];
    __shared__ double values[ANY ? kRows : 1][ANY ? kMost : 1];            // of the groups
    const int l = threadIdx.x % L, r = threadIdx.x / L, E = a.experts;
    const int64_t row = ((int64_t)from + blockIdx.x) * kRows + r;
    const bool live = row < a.N;
    if (a.load && from + blockIdx.x == 0) {                      // counted by the launch behind this one
        for (int e = threadIdx.x; e < E; e += kRouteThreads) a.load[e] = 0;
    }
    float x[V];
    double s[V], key[V];
    const int have = min(max(E - l * V, 0), V);                  // of the lane's experts
    load_logits(a.logits, row * a.ldl + l * V, live ? have : 0, a.t, x);
    float bias[V] = {};
    if (a.bias) load_run<SP24_F32>(a.bias, l * V, have, 0.0f, bias);
    scores_of_row<L>(x, a.softmax, s);
    // What is compared: a NaN is the largest, +inf (of a bias) the next; an expert that cannot be chosen is -inf.
    float rounded[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const double c = sum_of{}(s[i], (double)bias[i]);
        key[i] = x[i] == -__builtin_inff() ? kNever : c != c ? __builtin_inf() : __builtin_fmin(c, kInfinite);
        scores[r][i * L + l] = s[i];
        rounded[i] = (float)s[i];
    }
    if (a.scores && live) store_run<SP24_F32>(a.scores, row * E + l * V, have, rounded);
    if constexpr (GROUPS == kLaneGroups) {
        // the two largest of the lane, then of the lanes of its group
        double first = key[0], second = kNever;
#pragma unroll
        for (int i = 1; i < V; ++i) {
            second = __builtin_fmax(second, __builtin_fmin(first, key[i]));
            first = __builtin_fmax(first, key[i]);
        }
        const int lanes = E / a.groups / V;
        for (int d = 1; d < lanes; d *= 2) {
            const double other = __shfl_xor(first, d), next = __shfl_xor(second, d);
            second = __builtin_fmax(__builtin_fmin(first, other), __builtin_fmax(second, next));
            first = __builtin_fmax(first, other);
        }
        const double value = group_value(first, second, a.group_best);
        // the group stays if fewer than groups_kept are ahead of it
        const int mine = l / lanes;
        int ahead = 0;
        for (int h = 0; h < a.groups; ++h) {
            const double v = row_lane<L>(value, h * lanes);
            ahead += v > value || (v == value && h < mine);
        }
        if (ahead >= a.groups_kept) {
#pragma unroll
            for (int i = 0; i < V; ++i) key[i] = kNever;
        }
    }
    if constexpr (ANY) {
        const int size = E / a.groups;
#pragma unroll
        for (int i = 0; i < V; ++i) keys[r][i * L + l] = key[i];
        __syncthreads();
        for (int g = l; g < a.groups; g += L) {
            double first = kNever, second = kNever;
            for (int i = 0; i < size; ++i) {
                const double k = keys[r][image_place<L, V>(g * size + i)];
                second = __builtin_fmax(second, __builtin_fmin(first, k));
                first = __builtin_fmax(first, k);
            }
            values[r][g] = group_value(first, second, a.group_best);
        }
        __syncthreads();
        for (int g = l; g < a.groups; g += L) {
            const double mine = values[r][g];
            int ahead = 0;
            for (int h = 0; h < a.groups; ++h) ahead += values[r][h] > mine || (values[r][h] == mine && h < g);
            if (ahead >= a.groups_kept)
                for (int i = 0; i < size; ++i) keys[r][image_place<L, V>(g * size + i)] = kNever;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = keys[r][i * L + l];
    }
    // One after the other.  The row's largest is found by the lanes' best rounded to binary32, which keeps their order and takes one operation a step; where
    // two lanes are the same there, by all bits (reductions in binary64 always: 8192 rows, eight of 256, 11.2 us for 9.8, bf16 logits, which are often the same, 11.1
    // for 10.0).  A chosen one's upper half becomes that of a number below all others (the lower stays, so it is one word).
    uint32_t upper[V], lower[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint64_t bits = __builtin_bit_cast(uint64_t, key[i]);
        upper[i] = (uint32_t)(bits >> 32);
        lower[i] = (uint32_t)bits;
    }
    auto value = [&](int i) { return __builtin_bit_cast(double, ((uint64_t)upper[i] << 32) | lower[i]); };
    auto lane_best = [&] {
        double best = value(0);
#pragma unroll
        for (int i = 1; i < V; ++i) best = larger(best, value(i));
        return best;
    };
    double best = lane_best();
    for (int j = 0; j < a.topk; ++j) {
        const uint32_t small = in_order((float)best), most = most_of_row<L>(small);
        bool mine = small == most;
        const uint64_t have = __ballot(mine);
        if (__builtin_popcountll(have) > 64 / L) {
            const uint64_t full = __ballot(best == over_row<L>(best, larger_of{})) >> ((threadIdx.x & 63) / L * L);
            mine = l == __builtin_ctzll(full);                   // the lowest lane that has it, and there the lowest expert
        }
        if (mine) {
            int at = 0;
            bool found[V];
#pragma unroll
            for (int i = 0; i < V; ++i) found[i] = value(i) == best;
#pragma unroll
            for (int i = V - 1; i >= 0; --i) at = found[i] ? i : at;
#pragma unroll
            for (int i = 0; i < V; ++i) upper[i] = at == i ? kChosen : upper[i];
            picked[r][j] = most <= in_order(-__builtin_inff()) ? -1 : l * V + at;
            best = lane_best();
        }
    }
    __syncthreads();
    double chosen[kParts] = {};
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        if (i > 0 && i * L >= a.topk) break;
        const int j = i * L + l, e = j < a.topk ? picked[r][j] : -1;
        chosen[i] = e < 0 ? 0.0 : scores[r][image_place<L, V>(e)];
    }
    const double sum = sum_of_choices<L>(chosen, a.topk);
    if (!live) return;
    for (int j = l; j < a.topk; j += L) {
        const int e = picked[r][j];
        double w = e < 0 ? 0.0 : scores[r][image_place<L, V>(e)];
        if (a.renormalise) w = sum == 0.0 || e < 0 ? 0.0 : w / sum;
        a.ids[row * a.topk + j] = e;
        a.weights[row * a.topk + j] = (float)(w * (double)a.scale);
    }
}

// How many choices are each expert's: whole numbers, whose sums do not hang on their order.
constexpr int kLoadThreads = 1024, kLoadChoices = 4096;          // of a workgroup
__global__ __launch_bounds__(kLoadThreads) void k_route_load(const int32_t* ids, int32_t* load, int64_t choices, int experts)
{
    __shared__ int count[SP24_MOST_EXPERTS];
    for (int e = threadIdx.x; e < experts; e += kLoadThreads) count[e] = 0;
    __syncthreads();
    for (int64_t first = (int64_t)blockIdx.x * kLoadChoices; first < choices; first += (int64_t)gridDim.x * kLoadChoices) {
#pragma unroll
        for (int u = 0; u < kLoadChoices / kLoadThreads; ++u) {
            const int64_t i = first + u * kLoadThreads + threadIdx.x;
            const int e = i < choices ? ids[i] : -1;
            if (e >= 0) atomicAdd(&count[e], 1);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kLoadThreads)
        if (count[e] != 0) atomicAdd(load + e, count[e]);
}
__global__ void k_no_load(int32_t* load, int experts)
{
    for (int e = threadIdx.x; e < experts; e += blockDim.x) load[e] = 0;
}

template <int L, int V>
__global__ __launch_bounds__(kRouteThreads) void k_route_grad(RouteGradArgs a, unsigned from)
{
    constexpr int kRows = kRouteThreads / L, kMost = L * V, kPicks = kMost < SP24_MOST_CHOICES ? kMost : SP24_MOST_CHOICES;
    __shared__ double scores[kRows][kMost];
    __shared__ double slope[kRows][kPicks + 1];                  // of no choice (0), and of every one
    __shared__ int at[kRows][kPicks];
    __shared__ uint8_t choice[kRows][kMost];                     // an expert's, from 1 on, or 0
    const int l = threadIdx.x % L, r = threadIdx.x / L, E = a.experts;
    const int64_t row = ((int64_t)from + blockIdx.x) * kRows + r;
    const bool live = row < a.N;
    float x[V];
    float ds[V] = {};
    double s[V], rest[V], g[V];
    const int have = live ? min(max(E - l * V, 0), V) : 0;
    load_logits(a.logits, row * a.ldl + l * V, have, a.t, x);
    if (a.dscores) load_run<SP24_F32>(a.dscores, row * E + l * V, have, 0.0f, ds);
    scores_of_row<L>(x, a.softmax, s, rest);
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = (double)ds[i];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        scores[r][i * L + l] = s[i];
        choice[r][l * V + i] = 0;
    }
    if (l == 0) slope[r][0] = 0.0;
    __syncthreads();
    double total = 0.0, along = 0.0;
    for (int j = l; j < a.topk; j += L) {
        int e = live ? a.ids[row * a.topk + j] : -1;
        if (e < 0 || e >= E) e = -1;
        const double dw = e < 0 ? 0.0 : (double)a.dweights[row * a.topk + j], w = e < 0 ? 0.0 : scores[r][image_place<L, V>(e)];
        total += w;
        along += dw * w;
        at[r][j] = e;
        slope[r][j + 1] = dw;
        if (e >= 0) choice[r][e] = (uint8_t)(j + 1);
    }
    total = over_row<L>(total, sum_of{});
    along = over_row<L>(along, sum_of{});
    for (int j = l; j < a.topk; j += L) {
        const double dw = slope[r][j + 1];
        slope[r][j + 1] = (double)a.scale * (!a.renormalise ? dw : total == 0.0 ? 0.0 : (dw - along / total) / total);
    }
    __syncthreads();
    // Each expert looks its choice up; an expert that is there twice has the last one's number, and every choice is looked at (always: 8192 rows, eight of 256, 10.5 us for 9.0; 64 of 1024 36 for 10).
    bool twice = false;
    for (int j = l; j < a.topk; j += L) twice |= at[r][j] >= 0 && choice[r][at[r][j]] != j + 1;
    if (__any(twice)) {
        for (int j = 0; j < a.topk; ++j) {
            const int e = at[r][j] - l * V;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (e == i) g[i] += slope[r][j + 1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] += slope[r][choice[r][l * V + i]];
    }
    double mean = 0.0;
    if (a.softmax) {
#pragma unroll
        for (int i = 0; i < V; ++i) mean += x[i] == -__builtin_inff() ? 0.0 : g[i] * s[i];
        mean = over_row<L>(mean, sum_of{});
    }
    float d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = x[i] == -__builtin_inff() ? 0.0f : (float)(s[i] * (a.softmax ? g[i] - mean : rest[i] * g[i]));
    const int64_t to = row * a.lddl + l * V;
    if (a.t == SP24_F32) store_run<SP24_F32>(a.dlogits, to, have, d);
    else if (a.t == SP24_BF16) store_run<SP24_BF16>(a.dlogits, to, have, d);
    else store_run<SP24_F16>(a.dlogits, to, have, d);
}

// f(integral_constant lanes, integral_constant values a lane) for rows of this many experts.  Few rows are a wavefront each, whose chain of operations
// is the time; many share wavefronts, which issue the less for each.  In a graph, us, top 8 of 256: 512 rows on 64 lanes 4.9, on 32 5.8; 2048 5.3 and
// 5.8; 3000 6.4 and 6.5; 4096 7.4 and 6.6; 16384 19.4 and 15.8.  Top 6 of 64: 512 rows on 64 lanes 3.3, on 16 3.9; 2048 3.65 and 4.1; 8192 6.7 and 4.6.
template <class F>
static sp24_status by_experts(int experts, int64_t rows, F&& f)
{
    using std::integral_constant;
    auto with = [&](auto few_lanes, auto few_values, auto lanes, auto values) { return rows <= 2048 ? f(few_lanes, few_values) : f(lanes, values); };
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    const integral_constant<int, 8> eight;
    const integral_constant<int, 16> sixteen;
    const integral_constant<int, 32> half;
    const integral_constant<int, 64> all;
    if (experts <= 8) return f(eight, one);
    if (experts <= 16) return f(sixteen, one);
    if (experts <= 32) return with(half, one, sixteen, two);
    if (experts <= 64) return with(all, one, sixteen, four);
    if (experts <= 128) return with(all, two, half, four);
    if (experts <= 256) return with(all, four, half, eight);
    if (experts <= 512) return f(all, eight);
    return f(all, sixteen);
}

sp24_status launch_moe_route(const RouteArgs& a, hipStream_t st)
{
    if (a.N == 0) {
        if (!a.load) return SP24_OK;
        k_no_load<<<1, 256, 0, st>>>(a.load, a.experts);
        return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
    }
    const sp24_status s = by_experts(a.experts, a.N, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value, kRows = kRouteThreads / L;
        return launch_in_parts((a.N + kRows - 1) / kRows, kRouteThreads, [&](unsigned from, unsigned grid) {
            const int size = a.experts / a.groups;
            if (a.groups == 1) k_route<L, V, kNoGroups><<<grid, kRouteThreads, 0, st>>>(a, from);
            else if (size % V == 0 && ((size / V) & (size / V - 1)) == 0) k_route<L, V, kLaneGroups><<<grid, kRouteThreads, 0, st>>>(a, from);
            else k_route<L, V, kAnyGroups><<<grid, kRouteThreads, 0, st>>>(a, from);
        });
    });
    if (s != SP24_OK || !a.load) return s;
    const int64_t choices = a.N * a.topk;
    k_route_load<<<(unsigned)std::min<int64_t>((choices + kLoadChoices - 1) / kLoadChoices, 64), kLoadThreads, 0, st>>>(a.ids, a.load, choices, a.experts);
    return hipGetLastError() == hipSuccess ? SP24_OK : SP24_ERR_LAUNCH;
}

sp24_status launch_moe_route_grad(const RouteGradArgs& a, hipStream_t st)
{
    return by_experts(a.experts, a.N, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value, kRows = kRouteThreads / L;
        return launch_in_parts((a.N + kRows - 1) / kRows, kRouteThreads, [&](unsigned from, unsigned grid) {
            k_route_grad<L, V><<<grid, kRouteThreads, 0, st>>>(a, from);
        });
    });
}

} // namespace sp24
