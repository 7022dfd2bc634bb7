// Routing rules beyond the gate's softmax over the selection (Sec. 2.1): scores s of a token over E experts become
//   p   softmax over the experts that are there, or 1 / (1 + exp(-s))
//   c   p + bias (without a bias: the order of s), by which experts are chosen
//   groups of E / G experts, of which the best top_groups by their largest c or the sum of their two largest stay
//   idx the top_k largest c of what stays, equal ones the lower expert first;  w = p[idx], renormalised over the choice, scaled
// Which expert is chosen is a whole number and may not hang on how a sum was rounded: choices are those of c in double precision.
#include <climits>

#include "common.h"

namespace moe_ep {

namespace {

constexpr int kRtExperts = 512, kRtTopK = 64;
constexpr int kRtLaneExperts = kRtExperts / 64;

__device__ __forceinline__ double wave_max(double x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x = fmax(x, __shfl_xor(x, d, 64));
    return x;
}
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ int wave_min(int x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x = min(x, __shfl_xor(x, d, 64));
    return x;
}

// a score as the rule reads it: -inf for an expert that is not there (NaN, -inf or the type's lowest value), +inf as the largest number
template <bool BF16>
__device__ __forceinline__ float read_score(const void* row, int e)
{
    const float v = BF16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[e] << 16) : static_cast<const float*>(row)[e];
    const float lowest = BF16 ? __uint_as_float(0xff7f0000u) : -__FLT_MAX__;
    return v > lowest ? fminf(v, __FLT_MAX__) : -__builtin_inff();
}

// Weights of the n chosen experts, a lane per slot: p over the choice does not need p itself, and is taken relative to the
// largest score of the choice, so that it is there also where every p is too small for its type.
//   softmax: exp(s - m);  sigmoid: p = exp(min(s, 0)) / (1 + exp(-|s|)), exp(m) taken out of the numerator
// top, total: largest score and sum of exp(s - top) over the experts that are there (softmax without renormalising).
struct Weights { bool sigmoid, renorm; float scale; };
__device__ __forceinline__ float slot_weight(const Weights& r, float s, bool full, float best_chosen, float top, float total)
{
    if (!full) return 0.f;
    if (r.sigmoid) {
        const float m = r.renorm ? fminf(best_chosen, 0.f) : 0.f;
        return expf(fminf(s, 0.f) - m) / (1.0f + expf(-fabsf(s)));
    }
    return r.renorm ? expf(s - best_chosen) : expf(s - top) / total;
}

// One token by one wavefront, everything in double.  c: E doubles of LDS; slot_e: top_k integers of LDS.
template <bool BF16>
__device__ void route_token(const RouteArgs& a, long long t, int lane, double* c, int* slot_e)
{
    const int E = a.E, k = a.k, G = a.groups, S = E / G;
    const char* const row = static_cast<const char*>(a.scores) + t * a.stride * (BF16 ? 2 : 4);
    const bool live = !a.token_mask || a.token_mask[t] != 0;
    float s[kRtLaneExperts];
    double key[kRtLaneExperts];
    double top = -__builtin_inf();
#pragma unroll
    for (int i = 0; i < kRtLaneExperts; ++i) {
        const int e = lane + 64 * i;
        s[i] = -__builtin_inff();
        if (live && e < E) {
            const float b = a.bias ? a.bias[e] : 0.f;
            if (b > -__builtin_inff()) s[i] = read_score<BF16>(row, e);
        }
        top = fmax(top, (double)s[i]);
    }
    top = wave_max(top);
    const bool any = top > -__builtin_inf();
    double sum = 0.0;
    if (!a.sigmoid) {
#pragma unroll
        for (int i = 0; i < kRtLaneExperts; ++i) sum += s[i] > -__builtin_inff() ? exp((double)s[i] - top) : 0.0;
        sum = wave_sum(sum);
    }
    // c, or s where its order is c's
    const bool by_value = a.bias != nullptr, group_value = by_value || a.group_top2;
#pragma unroll
    for (int i = 0; i < kRtLaneExperts; ++i) {
        const int e = lane + 64 * i;
        key[i] = -__builtin_inf();
        double v = -__builtin_inf();
        if (s[i] > -__builtin_inff()) {
            v = s[i];
            if (group_value) v = a.sigmoid ? 1.0 / (1.0 + exp(-(double)s[i])) : exp((double)s[i] - top) / sum;
            if (by_value) v += (double)a.bias[e];
            key[i] = by_value ? v : (double)s[i];
        }
        if (G > 1 && e < E) c[e] = v;
    }
    if (G > 1) {
        wavefront_lds_order();
        double value = -__builtin_inf();
        if (lane < G) {
            double m1 = -__builtin_inf(), m2 = -__builtin_inf();
            for (int i = 0; i < S; ++i) {
                const double v = c[lane * S + i];
                if (v > m1) { m2 = m1; m1 = v; } else m2 = fmax(m2, v);
            }
            value = a.group_top2 && m2 > -__builtin_inf() ? m1 + m2 : m1;
        }
        wavefront_lds_order();
        int ahead = 0;
        for (int g = 0; g < G; ++g) {
            const double other = __shfl(value, g, 64);
            ahead += other > value || (other == value && g < lane);
        }
        const unsigned long long kept = __ballot(lane < G && value > -__builtin_inf() && ahead < a.top_groups);
#pragma unroll
        for (int i = 0; i < kRtLaneExperts; ++i) {
            const int e = lane + 64 * i;
            if (e < E && !((kept >> (e / S)) & 1)) key[i] = -__builtin_inf();
        }
    }
    for (int r = 0; r < k; ++r) {
        double best = key[0];
#pragma unroll
        for (int i = 1; i < kRtLaneExperts; ++i) best = fmax(best, key[i]);
        best = wave_max(best);
        int e = INT_MAX;
        if (best > -__builtin_inf()) {
#pragma unroll
            for (int i = kRtLaneExperts - 1; i >= 0; --i) e = key[i] == best ? lane + 64 * i : e;
            e = wave_min(e);
#pragma unroll
            for (int i = 0; i < kRtLaneExperts; ++i) key[i] = e == lane + 64 * i ? -__builtin_inf() : key[i];
        }
        if (lane == 0) slot_e[r] = e == INT_MAX ? -1 : e;
    }
    wavefront_lds_order();
    const int e = lane < k ? slot_e[lane] : -1;
    wavefront_lds_order();
    const bool full = e >= 0;
    const float se = full ? read_score<BF16>(row, e) : -__builtin_inff();
    float best_chosen = se;
#pragma unroll
    for (int d = 32; d; d >>= 1) best_chosen = fmaxf(best_chosen, __shfl_xor(best_chosen, d, 64));
    const Weights r{a.sigmoid, a.renorm, a.scale};
    float w = slot_weight(r, se, full, best_chosen, any ? (float)top : 0.f, (float)sum);
    if (a.renorm) {
        float total = w;
#pragma unroll
        for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d, 64);
        w = total > 0.f ? w / total : 0.f;
    }
    if (lane < k) {
        a.idx[t * k + lane] = e;
        a.w[t * k + lane] = w * a.scale;
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void route_exact_kernel(RouteArgs a)
{
    __shared__ double s_c[4][kRtExperts];
    __shared__ int s_slot[4][kRtTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long t = (long long)blockIdx.x * 4 + wave;
    if (t < a.T) route_token<BF16>(a, t, lane, s_c[wave], s_slot[wave]);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t s)
{
    if (a.T <= 0) return hipSuccess;
    if (a.E < 1 || a.E > kRtExperts || a.k < 1 || a.k > kRtTopK || a.groups < 1 || a.groups > 64 || a.E % a.groups) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(((long long)a.T + 3) / 4));
    if (a.bf16) hipLaunchKernelGGL(route_exact_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(route_exact_kernel<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace moe_ep
