// Routing rules beyond the gate's softmax over the selection (Sec. 2.1): scores s of a token over E experts become
//   p   softmax over the experts that are there, or 1 / (1 + exp(-s))
//   c   p + bias (without a bias: the order of s), by which experts are chosen
//   groups of E / G experts, of which the best top_groups by their largest c or the sum of their two largest stay
//   idx the top_k largest c of what stays, equal ones the lower expert first;  w = p[idx], renormalised over the choice, scaled
// Which expert is chosen is a whole number and may not hang on how a sum was rounded: choices are those of c in double precision.  Computing
// them so for every token (route_exact_kernel, a wavefront per token, also the kernel of shapes that the other one does not have) took 150 us
// for 65536 tokens of 256 experts.  route_kernel computes c in fp32 and looks whether two values that an order hangs on are closer than its
// rounding; chosen slots that are close are compared in double by the lanes that hold them.  A token is done again in double as a whole (5 us where it
// is the last one of a launch) only where its last slot or last group hangs on such a pair, where experts like the last that the list holds may come
// with it, or where two softmax values are a step of double apart.  The same 65536 tokens take 18 us, 36 with a bias, of which reading the scores is
// 14: instruction issue bounds it.
#include "gate.h"

namespace moe_ep {

namespace {

constexpr int kRtExperts = 512, kRtTopK = 64;
constexpr int kRtLaneExperts = kRtExperts / 64;
constexpr int kRtFewTokens = 8192;   // 16 lanes per token up to here (launch_route)

// the value of the lane that row_exchange names, of wider types
template <int CTRL>
__device__ __forceinline__ float exchange(float x) { return __int_as_float(row_exchange<CTRL>(__float_as_int(x))); }
template <int CTRL>
__device__ __forceinline__ int exchange(int x) { return row_exchange<CTRL>(x); }
template <int CTRL>
__device__ __forceinline__ double exchange(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)row_exchange<CTRL>((int)(uint32_t)u), hi = (uint32_t)row_exchange<CTRL>((int)(u >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// f over n lanes (a power of two up to 16) of every n: neighbours, pairs, then mirrors
template <class T, class F>
__device__ __forceinline__ T over_lanes(T x, int n, F f)
{
    if (n > 1) x = f(x, exchange<0xB1>(x));
    if (n > 2) x = f(x, exchange<0x4E>(x));
    if (n > 4) x = f(x, exchange<0x141>(x));
    if (n > 8) x = f(x, exchange<0x140>(x));
    return x;
}
// f over the wavefront: its rows of 16 lanes, then what their first lanes have
template <class T>
__device__ __forceinline__ T of_lane(T x, int lane)
{
    if constexpr (sizeof(T) == 8) {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, lane), hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), lane);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    } else return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}
template <class T, class F>
__device__ __forceinline__ T over_wave(T x, F f)
{
    x = over_lanes(x, 16, f);
    return f(f(of_lane(x, 0), of_lane(x, 16)), f(of_lane(x, 32), of_lane(x, 48)));
}
struct Most { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; } };
struct Least { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a < b ? a : b; } };
struct Plus { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a + b; } };

// a score as the rule reads it: -inf for an expert that is not there (NaN, -inf or the type's lowest value), +inf as the largest number
__device__ __forceinline__ float read_score(bool bf16, const void* row, int e)
{
    const float v = bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[e] << 16) : static_cast<const float*>(row)[e];
    const float lowest = bf16 ? __uint_as_float(0xff7f0000u) : -__FLT_MAX__;
    return v > lowest ? fminf(v, __FLT_MAX__) : -__builtin_inff();
}

// Weights of the n chosen experts, a lane per slot: p over the choice does not need p itself, and is taken relative to the
// largest score of the choice, so that it is there also where every p is too small for its type.
//   softmax: exp(s - m);  sigmoid: p = exp(min(s, 0)) / (1 + exp(-|s|)), exp(m) taken out of the numerator
// top, total: largest score and sum of exp(s - top) over the experts that are there (softmax without renormalising).
// In fp32: off by 5e-8 to 6e-8 (RMS, relative), twice what rounding a double once would be, and far less than the bf16 results that they weigh.
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

// One token by one wavefront, everything in double.  c: E doubles of LDS; slot_e: top_k integers of LDS.  In route_kernel a launch waits for the
// few tokens that come here: no exchange over the wavefront goes through LDS.
__device__ __forceinline__ void route_token(const RouteArgs& a, long long t, int lane, double* c, int* slot_e)
{
    const int E = a.E, k = a.k, G = a.groups, S = E / G;
    const double none = -__builtin_inf();
    const char* const row = static_cast<const char*>(a.scores) + t * a.stride * (a.bf16 ? 2 : 4);
    const bool live = !a.token_mask || a.token_mask[t] != 0;
    const bool by_value = a.bias != nullptr, group_value = by_value || a.group_top2;
    float s[kRtLaneExperts], b[kRtLaneExperts];
    double p[kRtLaneExperts], key[kRtLaneExperts];
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kRtLaneExperts; ++i) {
        const int e = lane + 64 * i;
        s[i] = -__builtin_inff();
        b[i] = 0.f;
        if (64 * i >= E) continue;
        if (live && e < E) {
            b[i] = by_value ? a.bias[e] : 0.f;
            if (b[i] > -__builtin_inff()) s[i] = read_score(a.bf16, row, e);
        }
        top = fmaxf(top, s[i]);
    }
    top = over_wave(top, Most());
    double sum = 0.0;
    if (!a.sigmoid && (group_value || !a.renorm)) {
#pragma unroll
        for (int i = 0; i < kRtLaneExperts; ++i) {
            p[i] = 0.0;
            if (64 * i < E && s[i] > -__builtin_inff()) p[i] = exp((double)s[i] - (double)top);
            sum += p[i];
        }
        sum = over_wave(sum, Plus());
    }
    // c, or s where its order is c's
#pragma unroll
    for (int i = 0; i < kRtLaneExperts; ++i) {
        key[i] = none;
        if (64 * i >= E) continue;
        double v = none;
        if (s[i] > -__builtin_inff()) {
            v = s[i];
            if (group_value) v = a.sigmoid ? 1.0 / (1.0 + exp(-(double)s[i])) : p[i] / sum;
            v += (double)b[i];
            key[i] = by_value ? v : (double)s[i];
        }
        if (G > 1 && lane + 64 * i < E) c[lane + 64 * i] = v;
    }
    if (G > 1) {
        wavefront_lds_order();
        // P lanes per group, a power of two up to 16
        const int P = G > 32 ? 1 : G > 16 ? 2 : G > 8 ? 4 : G > 4 ? 8 : 16, g = lane / P;
        double m1 = none, m2 = none;
        const auto take = [&](double v1, double v2) {
            const double low = v1 < m1 ? v1 : m1, high = v2 > m2 ? v2 : m2;
            m1 = v1 > m1 ? v1 : m1;
            m2 = low > high ? low : high;
        };
        if (g < G)
            for (int i = lane % P; i < S; i += P) take(c[g * S + i], none);
        if (P > 1) take(exchange<0xB1>(m1), exchange<0xB1>(m2));
        if (P > 2) take(exchange<0x4E>(m1), exchange<0x4E>(m2));
        if (P > 4) take(exchange<0x141>(m1), exchange<0x141>(m2));
        if (P > 8) take(exchange<0x140>(m1), exchange<0x140>(m2));
        wavefront_lds_order();
        const double value = g < G ? a.group_top2 && m2 > none ? m1 + m2 : m1 : none;
        int ahead = 0;
        for (int h = 0; h < G; ++h) {
            const double other = of_lane(value, h * P);
            ahead += other > value || (other == value && h < g);
        }
        const unsigned long long kept = __ballot(value > none && ahead < a.top_groups);   // a group's P lanes alike
#pragma unroll
        for (int i = 0; i < kRtLaneExperts; ++i) {
            const int e = lane + 64 * i;
            if (e < E && !((kept >> (e / S * P)) & 1)) key[i] = none;
        }
    }
    for (int r = 0; r < k; ++r) {
        double best = key[0];
#pragma unroll
        for (int i = 1; i < kRtLaneExperts; ++i)
            if (64 * i < E) best = key[i] > best ? key[i] : best;
        best = over_wave(best, Most());
        int e = INT_MAX;
        if (best > none) {
#pragma unroll
            for (int i = kRtLaneExperts - 1; i >= 0; --i)
                if (64 * i < E) e = key[i] == best ? lane + 64 * i : e;
            e = over_wave(e, Least());
#pragma unroll
            for (int i = 0; i < kRtLaneExperts; ++i) key[i] = e == lane + 64 * i ? none : key[i];
        }
        if (lane == 0) slot_e[r] = e == INT_MAX ? -1 : e;
    }
    wavefront_lds_order();
    const int e = lane < k ? slot_e[lane] : -1;
    wavefront_lds_order();
    const bool full = e >= 0;
    const float se = full ? read_score(a.bf16, row, e) : -__builtin_inff();
    const float best_chosen = over_wave(se, Most());
    const Weights r{a.sigmoid, a.renorm, a.scale};
    float w = slot_weight(r, se, full, best_chosen, top, (float)sum);
    if (a.renorm) {
        const float total = over_wave(w, Plus());
        w = total > 0.f ? w / total : 0.f;
    }
    if (lane < k) {
        a.idx[t * k + lane] = e;
        a.w[t * k + lane] = w * a.scale;
    }
}

// ---- the usual shapes: up to 16 experts per token, G a power of two up to the lanes of a token

// an expert as one number: its value's order (gate.h) in the upper bits, then the lower expert first; positive doubles that are no NaN have the
// order of their bits, and the f64 maximum and minimum run at the rate of fp32
__device__ __forceinline__ double ranked(float v, int behind)   // behind: kRtExperts - 1 - expert
{
    const uint32_t u = __float_as_uint(v + 0.0f), key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);   // v is no NaN
    return __builtin_bit_cast(double, (uint64_t)(key >> 2) << 32 | (key << 30 | (uint32_t)behind));
}
__device__ __forceinline__ float ranked_value(double x) { return key_score((uint32_t)(__builtin_bit_cast(uint64_t, x) >> 30)); }
__device__ __forceinline__ bool ranked_none(double x) { return (uint32_t)(__builtin_bit_cast(uint64_t, x) >> 32) <= 0x007fffffu >> 2; }   // -inf, or no expert at all
__device__ __forceinline__ int ranked_expert(double x) { return kRtExperts - 1 - (int)(__builtin_bit_cast(uint64_t, x) & (kRtExperts - 1)); }

__device__ __forceinline__ double larger(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double smaller(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ void in_order(double& a, double& b)
{
    const double x = larger(a, b);
    b = smaller(a, b);
    a = x;
}
// descending, by odd-even merges (Batcher)
template <int N>
__device__ __forceinline__ void sort(double (&a)[N])
{
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) in_order(a[i + j], a[i + j + k]);
}
// a: the N largest of both, descending as they were
template <int N>
__device__ __forceinline__ void merge(double (&a)[N], const double (&b)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = larger(a[i], b[N - 1 - i]);
#pragma unroll
    for (int d = N / 2; d; d /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(i & d)) in_order(a[i], a[i + d]);
}
template <int CTRL, int N>
__device__ __forceinline__ void merge_lanes(double (&a)[N])
{
    double b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) b[i] = exchange<CTRL>(a[i]);
    merge(a, b);
}
// A token is LANES lanes', each with REGS of its experts: of one group those of a group's lanes, VEC consecutive ones at a time.  The K
// best of a lane are sorted in registers, and the lanes' lists merged pair by pair: no round waits for another.  (A selection in rounds,
// a maximum over the lanes in each, waits for k of them.)  Instructions bound it where the tokens are many, 36 us of 65536 x 256 with a bias
// where the bytes are 14, and latency where they are few: 3.8 us of 256 tokens.
template <int LANES, int REGS, int K, int VEC, bool BIASED>
__global__ __launch_bounds__(256, !BIASED || REGS < 32 ? REGS * K <= 256 ? 4 : 3 : 2) void route_kernel(RouteArgs a)
{
    static_assert(K <= LANES && REGS % VEC == 0 && (REGS % K == 0 || REGS < K), "a slot per lane");
    __shared__ double s_c[4][kRtExperts];
    __shared__ int s_slot[4][kRtTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LANES;
    const long long t = (workgroup() * 4 + wave) * (64 / LANES) + lane / LANES;
    const int E = a.E, k = a.k, G = a.groups, S = E / G, LG = LANES / G, g = sub / LG;
    const bool there = t < a.T, live = there && (!a.token_mask || a.token_mask[t] != 0);
    const long long row_at = there ? t * a.stride : 0;   // a token that is not there reads the first one's scores
    const float none = -__builtin_inff();
    const int first = (sub % LG) * VEC;                  // inside the group; register r is expert first + (r / VEC) * LG * VEC + r % VEC
    float s[REGS], v[REGS];
    if (a.bf16) {
        const uint16_t* const row = static_cast<const uint16_t*>(a.scores) + row_at + g * S;
        typedef uint16_t v4 __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
        for (int r = 0; r < REGS; r += VEC) {
            const int m = first + r / VEC * (LG * VEC);
            if constexpr (VEC == 4) {
                v4 x = {0xffff, 0xffff, 0xffff, 0xffff};
                if (m < S) x = *reinterpret_cast<const v4*>(row + m);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[r + j] = __uint_as_float((uint32_t)x[j] << 16);
            } else s[r] = m < S ? __uint_as_float((uint32_t)row[m] << 16) : __uint_as_float(~0u);
        }
    } else {
        const float* const row = static_cast<const float*>(a.scores) + row_at + g * S;
        typedef float v4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int r = 0; r < REGS; r += VEC) {
            const int m = first + r / VEC * (LG * VEC);
            if constexpr (VEC == 4) {
                const float nan = __uint_as_float(~0u);
                v4 x = {nan, nan, nan, nan};
                if (m < S) x = *reinterpret_cast<const v4*>(row + m);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[r + j] = x[j];
            } else s[r] = m < S ? row[m] : __uint_as_float(~0u);
        }
    }
    constexpr bool by_value = BIASED;
    const bool group_value = by_value || a.group_top2;
    const float lowest = live ? a.bf16 ? __uint_as_float(0xff7f0000u) : -__FLT_MAX__ : __builtin_inff();
#pragma unroll
    for (int r = 0; r < REGS; ++r) s[r] = s[r] > lowest ? fminf(s[r], __FLT_MAX__) : none;
    if (by_value) {
        const float* const bias = a.bias + g * S;
        typedef float v4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int r = 0; r < REGS; r += VEC) {
            const int m = first + r / VEC * (LG * VEC);
            if constexpr (VEC == 4) {
                v4 x = {none, none, none, none};
                if (m < S) x = *reinterpret_cast<const v4*>(bias + m);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[r + j] = x[j];
            } else v[r] = m < S ? bias[m] : none;
        }
#pragma unroll
        for (int r = 0; r < REGS; ++r) s[r] = v[r] > none ? s[r] : none;
    }
    float top = 0.f, total = 0.f;
    if (!a.sigmoid && (group_value || !a.renorm)) {
        top = s[0];
#pragma unroll
        for (int r = 1; r < REGS; ++r) top = fmaxf(top, s[r]);
        top = over_lanes(top, LANES, Most());
        top = top > none ? top : 0.f;
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < REGS; ++r) part[r & 3] += __builtin_amdgcn_exp2f((s[r] - top) * 1.4426950408889634f);
        total = over_lanes((part[0] + part[1]) + (part[2] + part[3]), LANES, Plus());
    }
    // v: c; s itself where its order is asked for
    if (group_value) {
        const float by = total > 0.f ? __builtin_amdgcn_rcpf(total) : 0.f;
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const float p = a.sigmoid ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[r] * -1.4426950408889634f))
                                      : __builtin_amdgcn_exp2f((s[r] - top) * 1.4426950408889634f) * by;
            v[r] = s[r] > none ? by_value ? p + v[r] : p : none;
        }
    } else {
#pragma unroll
        for (int r = 0; r < REGS; ++r) v[r] = s[r];
    }
    // Two values that close may be in the other order.  Of a sigmoid p is off by less than 2^-22 (exp2, its argument, a sum, the reciprocal); of a softmax the
    // difference of two by 2^-21 and by 2^-19.3 of itself (their sum: 14 roundings in a row, and the arguments' of exponentials); c by half a step.  Twice all that (of a softmax 1.88 times).
    const float slack = a.sigmoid ? 0x1p-20f : 0x1p-18f;
    const auto close = [=](float x, float y, float by) { return x > none && y > none && !(fabsf(x - y) > by + 0x1p-22f * fmaxf(fabsf(x), fabsf(y))); };
    bool unsure = false;
    if (G > 1) {
        float m1 = v[0], m2 = none;
#pragma unroll
        for (int r = 1; r < REGS; ++r) {
            m2 = fmaxf(m2, fminf(m1, v[r]));
            m1 = fmaxf(m1, v[r]);
        }
        const auto both = [&](float o1, float o2) {
            m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
            m1 = fmaxf(m1, o1);
        };
        if (LG > 1) both(exchange<0xB1>(m1), exchange<0xB1>(m2));
        if (LG > 2) both(exchange<0x4E>(m1), exchange<0x4E>(m2));
        if (LG > 4) both(exchange<0x141>(m1), exchange<0x141>(m2));
        const float value = a.group_top2 && m2 > none ? m1 + m2 : m1;
        int ahead = 0;
        for (int h = 0; h < G; ++h) {
            const float other = __shfl(value, (lane & ~(LANES - 1)) + h * LG, 64);
            ahead += other > value || (other == value && h < g);
        }
        const bool stays = ahead < a.top_groups;   // (of a group without an expert every value says so)
        unsure = m1 > none && fabsf(m1) < __builtin_inff() && !(fabsf(value) < __builtin_inff());   // a sum that is beyond fp32, not beyond double
        // An order hangs on the last group that stays and the first that does not, each off by `off` at most: a p or two (half the slack, and half of that
        // again), and the steps of the two numbers, of their sum, which may be far smaller than they are, and of the sum with `off` (2^-24 of both, three times).
        const float off = m1 < __builtin_inff() ? 0.75f * slack + 0x1.9p-23f * fabsf(m1) + (a.group_top2 && m2 > none ? 0x1.9p-23f * fabsf(m2) : 0.f) : 0.f;
        if (group_value)
            unsure |= over_lanes(stays && value > none ? value - off : __builtin_inff(), LANES, Least()) <= over_lanes(!stays && value > none ? value + off : none, LANES, Most());
        if (!stays) {
#pragma unroll
            for (int r = 0; r < REGS; ++r) v[r] = s[r] = none;
        }
    }
    // without a bias experts are in the order of s
    if (!by_value) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) v[r] = s[r];
    }
    double list[K];
    const int behind = kRtExperts - 1 - (g * S + first);
    if constexpr (REGS <= K) {
#pragma unroll
        for (int r = 0; r < K; ++r) list[r] = r < REGS ? ranked(v[r < REGS ? r : 0], behind - (r / VEC * (LG * VEC) + r % VEC)) : 0.0;
        sort(list);
    } else {
#pragma unroll
        for (int b = 0; b < REGS; b += K) {
            double next[K];
#pragma unroll
            for (int r = 0; r < K; ++r) next[r] = ranked(v[b + r], behind - ((b + r) / VEC * (LG * VEC) + (b + r) % VEC));
            sort(next);
            if (b == 0) {
#pragma unroll
                for (int r = 0; r < K; ++r) list[r] = next[r];
            } else merge(list, next);
        }
    }
    merge_lanes<0xB1>(list);
    merge_lanes<0x4E>(list);
    merge_lanes<0x141>(list);
    if (LANES > 8) merge_lanes<0x140>(list);

    // a slot per lane, up to K: those from k on may still move up
    double mine = 0.0;
#pragma unroll
    for (int i = 0; i < K; ++i) mine = sub == i ? list[i] : mine;
    bool full = sub < K && !ranked_none(mine);
    int e = full ? ranked_expert(mine) : -1, place = sub;
    const auto score_of = [&](int expert) { return read_score(a.bf16, static_cast<const char*>(a.scores) + row_at * (a.bf16 ? 2 : 4), expert); };
    float se = none;
    if (full) se = by_value ? score_of(e) : ranked_value(mine);
    if constexpr (by_value) {
        // an order hangs on neighbouring slots, unless they are alike, and on the last slot and every expert behind it
        const float value = full ? ranked_value(mine) : none, be = full ? a.bias[e] : 0.f;
        const int base = lane & ~(LANES - 1), next = lane + 1;
        const float nv = __shfl(value, next, 64), ns = __shfl(se, next, 64), nb = __shfl(be, next, 64);
        const float lv = __shfl(value, base + k - 1, 64);
        float line = lv > none ? lv - (slack + 0x1p-21f * fabsf(lv)) : __builtin_inff();   // a last slot that is empty has nobody behind it
        line = line < -__FLT_MAX__ ? -__FLT_MAX__ : line;   // nor are those that are not there behind one whose bias is the lowest number
        bool near = (sub < k || value >= line) && sub + 1 < K && close(value, nv, slack) && !(se == ns && be == nb);
        int found = 0;
#pragma unroll
        for (int r = 0; r < REGS; ++r) found += __popcll(__ballot(v[r] >= line));
        double extra = 0.0;   // the best of those that are no slot
        bool alike = false;   // there are some like the last slot, which come right behind it
        if (found > __popcll(__ballot(full && value >= line))) {   // of some token of the wavefront: look which
            const int le = __shfl(e, base + K - 1, 64);
            const float ls = __shfl(se, base + K - 1, 64), lb = __shfl(be, base + K - 1, 64);
            int others = 0;
#pragma unroll
            for (int r = 0; r < REGS; ++r) {
                const int at = behind - (r / VEC * (LG * VEC) + r % VEC), other = kRtExperts - 1 - at;
                if (!(v[r] >= line)) continue;
                const double x = ranked(v[r], at);
                if (!(x < list[K - 1])) continue;
                if (le >= 0 && other > le && a.bias[other] == lb && score_of(other) == ls) {
                    alike = true;
                    continue;
                }
                extra = larger(extra, x);
                ++others;
            }
            alike = over_lanes((int)alike, LANES, Most()) != 0;
            extra = over_lanes(extra, LANES, [](double x, double y) { return larger(x, y); });
            others = over_lanes(others, LANES, Plus());
            near = near || others > 0;
            unsure = unsure || others > 1;
        }
        if (__ballot(near)) {
            // The slots' own values in double, of all tokens at once, and their order; the one in front of which all K are gives way to the other.
            // A softmax's sum stays in fp32: it is the same for both, so that the difference of two p is off by less than 2^-18 of itself, and two c that are
            // equal, or all but equal, may not have been rounded as they would with the sum in double.
            const auto p_of = [&](float score) { return a.sigmoid ? 1.0 / (1.0 + exp(-(double)score)) : exp((double)score - (double)top) / (double)total; };
            double p = 0.0, c = -__builtin_inf(), p_extra = 0.0, c_extra = -__builtin_inf();
            if (full) { p = p_of(se); c = p + (double)be; }
            int e_extra = -1, place_extra = 0;
            float s_extra = none, b_extra = 0.f;
            if (extra > 0.0) {
                e_extra = ranked_expert(extra);
                s_extra = score_of(e_extra);
                p_extra = p_of(s_extra);
                b_extra = a.bias[e_extra];
                c_extra = p_extra + (double)b_extra;
            }
            const auto ahead_of = [](double x, int ex, double y, int ey) { return x > y || (x == y && ex < ey); };
            const auto unclear = [&](double px, float bx, double x, double py, float by, double y) {
                return !a.sigmoid && (px != py || bx != by) && fabs(x - y) <= 0x1p-18 * fabs(px - py) + 0x1p-50 * fmin(fmax(fabs(x), px), fmax(fabs(y), py));
            };
            place = 0;
#pragma unroll 1
            for (int i = 0; i < K; ++i) {
                const int oe = __shfl(e, base + i, 64);
                const double op = __shfl(p, base + i, 64), oc = __shfl(c, base + i, 64);
                const float ob = __shfl(be, base + i, 64);
                if (oe < 0) continue;
                place += !full || ahead_of(oc, oe, c, e);   // empty slots stay behind
                place_extra += ahead_of(oc, oe, c_extra, e_extra);
                unsure = unsure || (full && unclear(op, ob, oc, p, be, c)) || (e_extra >= 0 && unclear(op, ob, oc, p_extra, b_extra, c_extra));
            }
            unsure = unsure || (alike && sub == K - 1 && place + 1 < k);
            if (!full) place = sub;
            else if (e_extra >= 0) {
                place += ahead_of(c_extra, e_extra, c, e);
                if (place == K) { e = e_extra; se = s_extra; place = place_extra; }
            }
        }
    }
    full = full && place < k;
    if (!full) se = none;
    const Weights rule{a.sigmoid, a.renorm, a.scale};
    const float best_chosen = over_lanes(se, LANES, Most());
    float w = slot_weight(rule, se, full, best_chosen, top, total);
    if (a.renorm) {
        const float sum = over_lanes(w, LANES, Plus());
        w = sum > 0.f ? w / sum : 0.f;
    }
    unsigned long long again = __ballot(unsure && there);
    constexpr unsigned long long TOKEN = (1ull << LANES) - 1ull;
    if (there && sub < K && place < k && !((again >> (lane & ~(LANES - 1))) & TOKEN)) {
        a.idx[t * k + place] = full ? e : -1;
        a.w[t * k + place] = w * a.scale;
    }
    while (again) {   // a token at a time, by the whole wavefront
        const int from = __builtin_ctzll(again) & ~(LANES - 1);
        again &= ~(TOKEN << from);
        const long long token = t - lane / LANES + from / LANES;
        route_token(a, token, lane, s_c[wave], s_slot[wave]);
        wavefront_lds_order();
    }
}

template <int LANES, int REGS, int K, int VEC>
hipError_t launch(const RouteArgs& a, hipStream_t s)
{
    const long long tokens = 4 * (64 / LANES);
    const dim3 grid = grid_of(((long long)a.T + tokens - 1) / tokens);
    if (a.bias) hipLaunchKernelGGL((route_kernel<LANES, REGS, K, VEC, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((route_kernel<LANES, REGS, K, VEC, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int LANES, int K, int VEC>
hipError_t launch_regs(const RouteArgs& a, int regs, hipStream_t s)
{
    if (regs <= 8) return launch<LANES, 8, K, VEC>(a, s);
    return regs <= 16 ? launch<LANES, 16, K, VEC>(a, s) : launch<LANES, 32, K, VEC>(a, s);
}

// ---- every shape

__global__ __launch_bounds__(256) void route_exact_kernel(RouteArgs a)
{
    __shared__ double s_c[4][kRtExperts];
    __shared__ int s_slot[4][kRtTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long t = workgroup() * 4 + wave;
    if (t < a.T) route_token(a, t, lane, s_c[wave], s_slot[wave]);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t s)
{
    if (a.T <= 0) return hipSuccess;
    if (a.E < 1 || a.E > kRtExperts || a.k < 1 || a.k > kRtTopK || a.groups < 1 || a.groups > 64 || a.E % a.groups) return hipErrorInvalidValue;
    // registers a lane needs with `lanes` lanes per token, VEC experts at a time
    const bool groups_fit = (a.groups & (a.groups - 1)) == 0 && a.groups <= 16;
    const int size = a.E / a.groups, vec = size % 4 == 0 ? 4 : 1;
    const auto regs = [&](int lanes) { return (size + lanes / a.groups * vec - 1) / (lanes / a.groups * vec) * vec; };
    if (groups_fit && a.k <= 16) {
        // 8 lanes a token sort and merge less in all, 16 lanes are shorter.  8 / 16, us, 256 experts: 4096 tokens 4.5 / 4.0, 8192 4.6 / 4.7,
        // 65536 19.7 / 20.9; 128 with a bias: 4096 7.4 / 5.8, 8192 7.4 / 7.5, 65536 18.8 / 23.7; 160 in 8 groups 5.3 / 4.7, 5.4 / 5.4, 20 / 24.
        // 64 experts: 512 3.3 / 3.4, 65536 9.1 / 15.5.  32 experts a lane with a bias, which keeps p and c, spill: 65536 35 / 31.
        if (a.k <= 8 && a.groups <= 8 && regs(8) <= (a.bias ? 16 : 32) && (a.T > kRtFewTokens || (!a.bias && regs(8) <= 8)))
            return vec == 4 ? launch_regs<8, 8, 4>(a, regs(8), s) : launch_regs<8, 8, 1>(a, regs(8), s);
        if (regs(16) <= 32) {
            if (a.k <= 8) return vec == 4 ? launch_regs<16, 8, 4>(a, regs(16), s) : launch_regs<16, 8, 1>(a, regs(16), s);
            return vec == 4 ? launch_regs<16, 16, 4>(a, regs(16), s) : launch_regs<16, 16, 1>(a, regs(16), s);
        }
    }
    const dim3 grid = grid_of(((long long)a.T + 3) / 4);
    hipLaunchKernelGGL(route_exact_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace moe_ep
