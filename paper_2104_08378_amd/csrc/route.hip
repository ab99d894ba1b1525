// The experts of every token from the router's logits, and the gradient of what comes of it.
//
//   s = softmax(l) or 1 / (1 + e^-l),  c = s + bias;  the experts of the largest c, their weights s / sum s (or s) times scale
//   g[e] = ds[e] + sum over j of [ids[j] = e] dg[j],  dg = scale (dw - sum(dw s) / W) / W  (not renormalised: scale dw),  W = sum of the chosen s
//   softmax: dl = s (g - sum g s);  logistic: dl = s (1 - s) g
//
// All in binary64: of 10^5 tokens' experts some pairs' scores are within a rounding of binary32 of each other, and which one is chosen must
// not hang on the order of a sum.
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
// OP over the L lanes of a row, the same in all of them and in the same order always
template <int L, class OP>
__device__ __forceinline__ double over_row(double v, OP op)
{
    if constexpr (L >= 2) v = op(v, dpp_of<0xB1>(v));            // quad_perm [1,0,3,2]
    if constexpr (L >= 4) v = op(v, dpp_of<0x4E>(v));            // quad_perm [2,3,0,1]
    if constexpr (L >= 8) v = op(v, dpp_of<0x141>(v));           // the other half of eight lanes, mirrored
    if constexpr (L >= 16) v = op(v, dpp_of<0x140>(v));          // the other half of sixteen
    if constexpr (L >= 32) v = op(v, __shfl_xor(v, 16));
    if constexpr (L >= 64) v = op(v, __shfl_xor(v, 32));
    return v;
}
struct larger_of { __device__ __forceinline__ double operator()(double a, double b) const { return __builtin_fmax(a, b); } };
struct sum_of { __device__ __forceinline__ double operator()(double a, double b) const { return a + b; } };

__device__ __forceinline__ float logit_of(const void* p, int64_t i, sp24_dtype t)
{
    return t == SP24_F32 ? load_value<SP24_F32>(p, i) : t == SP24_BF16 ? load_value<SP24_BF16>(p, i) : load_value<SP24_F16>(p, i);
}

constexpr double kNever = -__builtin_inf();

// The scores of a row's experts, 0 for those whose logit is -inf.  A NaN (or, softmax, +inf) makes NaN of what it takes part in.
template <int L, int V>
__device__ __forceinline__ void scores_of_row(const float (&x)[V], bool softmax, double (&s)[V])
{
    if (softmax) {
        float most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < V; ++i) most = fmaxf(most, x[i]);
        const double top = over_row<L>((double)most, larger_of{});
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[i] = x[i] == -__builtin_inff() ? 0.0 : exp((double)x[i] - top);
            sum += s[i];
        }
        sum = over_row<L>(sum, sum_of{});
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = x[i] == -__builtin_inff() ? 0.0 : s[i] / sum;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = x[i] == -__builtin_inff() ? 0.0 : 1.0 / (1.0 + exp(-(double)x[i]));
    }
}

template <int L, int V, bool GROUPS>
__global__ __launch_bounds__(kRouteThreads) void k_route(RouteArgs a, unsigned from)
{
    constexpr int kRows = kRouteThreads / L, kMost = L * V, kPicks = kMost < SP24_MOST_CHOICES ? kMost : SP24_MOST_CHOICES;
    __shared__ double picked_s[kRows][kPicks];
    __shared__ int picked_e[kRows][kPicks];
    __shared__ double keys[GROUPS ? kRows : 1][GROUPS ? kMost : 1];
    __shared__ double values[GROUPS ? kRows : 1][GROUPS ? kMost : 1];      // of the groups; then whether they stay
    const int l = threadIdx.x % L, r = threadIdx.x / L, E = a.experts;
    const int64_t row = ((int64_t)from + blockIdx.x) * kRows + r;
    const bool live = row < a.N;
    float x[V];
    double s[V], key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = live && l * V + i < E ? logit_of(a.logits, row * a.ldl + l * V + i, a.t) : -__builtin_inff();
    scores_of_row<L>(x, a.softmax, s);
    // What is compared: a NaN is the largest, +inf (of a bias) the next; an expert that cannot be chosen is -inf.
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = l * V + i;
        const double c = s[i] + (a.bias && e < E ? (double)a.bias[e] : 0.0);
        key[i] = x[i] == -__builtin_inff() ? kNever : c != c ? __builtin_inf() : __builtin_fmin(c, 1e300);
        if (a.scores && live && e < E) a.scores[row * E + e] = (float)s[i];
    }
    if constexpr (GROUPS) {
        const int size = E / a.groups;
#pragma unroll
        for (int i = 0; i < V; ++i) keys[r][l * V + i] = key[i];
        __syncthreads();
        for (int g = l; g < a.groups; g += L) {
            double first = kNever, second = kNever;
            for (int i = 0; i < size; ++i) {
                const double k = keys[r][g * size + i];
                second = __builtin_fmax(second, __builtin_fmin(first, k));
                first = __builtin_fmax(first, k);
            }
            values[r][g] = a.group_best == 1 || second == kNever ? first : first + second;
        }
        __syncthreads();
        // a group stays if fewer than groups_kept are ahead of it
        for (int i = 0; i < V; ++i) {
            const int g = l * V + i < E ? (l * V + i) / size : 0;
            const double mine = values[r][g];
            int ahead = 0;
            for (int h = 0; h < a.groups; ++h) ahead += values[r][h] > mine || (values[r][h] == mine && h < g);
            if (ahead >= a.groups_kept) keys[r][l * V + i] = kNever;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = keys[r][l * V + i];
    }
    for (int j = 0; j < a.topk; ++j) {
        double best = key[0];
#pragma unroll
        for (int i = 1; i < V; ++i) best = __builtin_fmax(best, key[i]);
        const double most = over_row<L>(best, larger_of{});
        const uint64_t have = __ballot(best == most) >> ((threadIdx.x & 63) / L * L);
        const bool none = most == kNever;
        if (l == __builtin_ctzll(have)) {                        // the lowest lane that has it, and there the lowest expert
            int at = -1;
            double score = 0.0;
#pragma unroll
            for (int i = V - 1; i >= 0; --i)
                if (key[i] == most) {
                    at = i;
                    score = s[i];
                }
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i == at) key[i] = kNever;
            picked_e[r][j] = none ? -1 : l * V + at;
            picked_s[r][j] = none ? 0.0 : score;
        }
    }
    __syncthreads();
    double sum = 0.0;
    for (int j = l; j < a.topk; j += L) sum += picked_s[r][j];
    sum = over_row<L>(sum, sum_of{});
    if (!live) return;
    for (int j = l; j < a.topk; j += L) {
        const int e = picked_e[r][j];
        double w = picked_s[r][j];
        if (a.renormalise && e >= 0) w = sum == 0.0 ? 0.0 : w / sum;
        a.ids[row * a.topk + j] = e;
        a.weights[row * a.topk + j] = e < 0 ? 0.0f : (float)(w * (double)a.scale);
        if (a.load && e >= 0) atomicAdd(a.load + e, 1);
    }
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
    __shared__ double slope[kRows][kPicks];
    __shared__ int at[kRows][kPicks];
    const int l = threadIdx.x % L, r = threadIdx.x / L, E = a.experts;
    const int64_t row = ((int64_t)from + blockIdx.x) * kRows + r;
    const bool live = row < a.N;
    float x[V];
    double s[V], g[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = l * V + i;
        x[i] = live && e < E ? logit_of(a.logits, row * a.ldl + e, a.t) : -__builtin_inff();
        g[i] = a.dscores && live && e < E ? (double)a.dscores[row * E + e] : 0.0;
    }
    scores_of_row<L>(x, a.softmax, s);
#pragma unroll
    for (int i = 0; i < V; ++i) scores[r][l * V + i] = s[i];
    __syncthreads();
    double total = 0.0, along = 0.0;
    for (int j = l; j < a.topk; j += L) {
        int e = live ? a.ids[row * a.topk + j] : -1;
        if (e < 0 || e >= E) e = -1;
        const double dw = e < 0 ? 0.0 : (double)a.dweights[row * a.topk + j], w = e < 0 ? 0.0 : scores[r][e];
        total += w;
        along += dw * w;
        at[r][j] = e;
        slope[r][j] = dw;
    }
    total = over_row<L>(total, sum_of{});
    along = over_row<L>(along, sum_of{});
    for (int j = l; j < a.topk; j += L) {
        const double dw = slope[r][j];
        slope[r][j] = (double)a.scale * (!a.renormalise ? dw : total == 0.0 ? 0.0 : (dw - along / total) / total);
    }
    __syncthreads();
    for (int j = 0; j < a.topk; ++j) {
        const int e = at[r][j] - l * V;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (e == i) g[i] += slope[r][j];
    }
    double mean = 0.0;
    if (a.softmax) {
#pragma unroll
        for (int i = 0; i < V; ++i) mean += x[i] == -__builtin_inff() ? 0.0 : g[i] * s[i];
        mean = over_row<L>(mean, sum_of{});
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = l * V + i;
        if (e >= E) continue;
        const double d = x[i] == -__builtin_inff() ? 0.0 : s[i] * (a.softmax ? g[i] - mean : (1.0 - s[i]) * g[i]);
        const int64_t to = row * a.lddl + e;
        if (a.t == SP24_F32) store_out<SP24_F32>(a.dlogits, to, (float)d);
        else if (a.t == SP24_BF16) store_out<SP24_BF16>(a.dlogits, to, (float)d);
        else store_out<SP24_F16>(a.dlogits, to, (float)d);
    }
}

// f(integral_constant lanes, integral_constant values a lane) for a row of this many experts
template <class F>
static sp24_status by_experts(int experts, F&& f)
{
    auto with = [&](auto l, auto v) { return f(l, v); };
    using std::integral_constant;
    if (experts <= 8) return with(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (experts <= 16) return with(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (experts <= 32) return with(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (experts <= 64) return with(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (experts <= 128) return with(integral_constant<int, 32>{}, integral_constant<int, 4>{});
    if (experts <= 256) return with(integral_constant<int, 32>{}, integral_constant<int, 8>{});
    if (experts <= 512) return with(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    return with(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

sp24_status launch_moe_route(const RouteArgs& a, hipStream_t st)
{
    if (a.load) k_no_load<<<1, 256, 0, st>>>(a.load, a.experts);
    return by_experts(a.experts, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value, kRows = kRouteThreads / L;
        return launch_in_parts((a.N + kRows - 1) / kRows, kRouteThreads, [&](unsigned from, unsigned grid) {
            if (a.groups > 1) k_route<L, V, true><<<grid, kRouteThreads, 0, st>>>(a, from);
            else k_route<L, V, false><<<grid, kRouteThreads, 0, st>>>(a, from);
        });
    });
}

sp24_status launch_moe_route_grad(const RouteGradArgs& a, hipStream_t st)
{
    return by_experts(a.experts, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value, kRows = kRouteThreads / L;
        return launch_in_parts((a.N + kRows - 1) / kRows, kRouteThreads, [&](unsigned from, unsigned grid) {
            k_route_grad<L, V><<<grid, kRouteThreads, 0, st>>>(a, from);
        });
    });
}

} // namespace sp24
