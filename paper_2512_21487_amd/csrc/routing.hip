// Routing rules beyond the gate's softmax over the selection (Sec. 2.1): scores s of a token over E experts become
//   p   softmax over the experts that are there, or 1 / (1 + exp(-s))
//   c   p + bias (without a bias: the order of s), by which experts are chosen
//   groups of E / G experts, of which the best top_groups by their largest c or the sum of their two largest stay
//   idx the top_k largest c of what stays, equal ones the lower expert first;  w = p[idx], renormalised over the choice, scaled
// Which expert is chosen is a whole number and may not hang on how a sum was rounded: choices are those of c in double precision.  Computing
// them so for every token (route_exact_kernel, a wavefront per token, also the kernel of shapes that the other one does not have) took 150 us
// for 65536 tokens of 256 experts.  route_kernel computes c in fp32 and looks whether two values that an order hangs on are closer than its
// rounding; of normal scores about one token in a thousand is such, and is done again in double.
#include "gate.h"

namespace moe_ep {

namespace {

constexpr int kRtExperts = 512, kRtTopK = 64;
constexpr int kRtLaneExperts = kRtExperts / 64;
constexpr int kRtFewTokens = 2048;   // 16 lanes per token up to here: more wavefronts, and shorter ones

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
__device__ __forceinline__ void route_token(const RouteArgs& a, long long t, int lane, double* c, int* slot_e)
{
    const int E = a.E, k = a.k, G = a.groups, S = E / G;
    const char* const row = static_cast<const char*>(a.scores) + t * a.stride * (a.bf16 ? 2 : 4);
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
            if (b > -__builtin_inff()) s[i] = read_score(a.bf16, row, e);
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
    const float se = full ? read_score(a.bf16, row, e) : -__builtin_inff();
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

// ---- the usual shapes: up to 16 experts per token, G a power of two up to the lanes of a token

// an expert as one number: its value's order (gate.h) in the upper bits, then the lower expert first; positive doubles that are no NaN have the
// order of their bits, and the f64 maximum and minimum run at the rate of fp32
__device__ __forceinline__ double ranked(float v, int e)
{
    const uint32_t key = v > -__builtin_inff() ? order_key(v) : 0u;
    const uint64_t bits = (uint64_t)(key >> 2) << 32 | (key ? key << 30 | (uint32_t)(kRtExperts - 1 - e) : 0u);
    return __builtin_bit_cast(double, bits);
}
__device__ __forceinline__ bool ranked_none(double x) { return __builtin_bit_cast(uint64_t, x) == 0; }
__device__ __forceinline__ int ranked_expert(double x) { return kRtExperts - 1 - (int)(__builtin_bit_cast(uint64_t, x) & (kRtExperts - 1)); }
__device__ __forceinline__ float ranked_value(double x) { return key_score((uint32_t)(__builtin_bit_cast(uint64_t, x) >> 30)); }

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
template <int CTRL>
__device__ __forceinline__ float exchange(float x) { return __int_as_float(row_exchange<CTRL>(__float_as_int(x))); }
template <int CTRL>
__device__ __forceinline__ double exchange(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)row_exchange<CTRL>((int)(uint32_t)u), hi = (uint32_t)row_exchange<CTRL>((int)(u >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL, int N>
__device__ __forceinline__ void merge_lanes(double (&a)[N])
{
    double b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) b[i] = exchange<CTRL>(a[i]);
    merge(a, b);
}
// over the first n (a power of two) lanes of every n: neighbours, pairs, then mirrors
template <class F>
__device__ __forceinline__ float over_lanes(float x, int n, F f)
{
    if (n > 1) x = f(x, exchange<0xB1>(x));
    if (n > 2) x = f(x, exchange<0x4E>(x));
    if (n > 4) x = f(x, exchange<0x141>(x));
    if (n > 8) x = f(x, exchange<0x140>(x));
    return x;
}

// A token is LANES lanes', each with REGS of its experts: of one group those of a group's lanes, VEC consecutive ones at a time.  The K
// best of a lane are sorted in registers, and the lanes' lists merged pair by pair: no round waits for another.  What bounds it is the
// instructions, about 50 a token (8 lanes, 32 experts a lane), and the scores' bytes close behind.
template <int LANES, int REGS, int K, int VEC>
__global__ __launch_bounds__(256, REGS * K <= 256 ? 4 : 3) void route_kernel(RouteArgs a)
{
    static_assert(K <= LANES && REGS % VEC == 0 && (REGS % K == 0 || REGS < K), "a slot per lane");
    __shared__ double s_c[4][kRtExperts];
    __shared__ int s_slot[4][kRtTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LANES;
    const long long t = ((long long)blockIdx.x * 4 + wave) * (64 / LANES) + lane / LANES;
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
    const bool by_value = a.bias != nullptr, group_value = by_value || a.group_top2;
    const float lowest = live ? a.bf16 ? __uint_as_float(0xff7f0000u) : -__FLT_MAX__ : __builtin_inff();
    if (by_value) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const int m = first + r / VEC * (LG * VEC) + r % VEC;
            v[r] = m < S ? a.bias[g * S + m] : none;
        }
#pragma unroll
        for (int r = 0; r < REGS; ++r) s[r] = s[r] > lowest && v[r] > none ? fminf(s[r], __FLT_MAX__) : none;
    } else {
#pragma unroll
        for (int r = 0; r < REGS; ++r) s[r] = s[r] > lowest ? fminf(s[r], __FLT_MAX__) : none;
    }
    const auto most = [](float x, float y) { return fmaxf(x, y); };
    const auto plus = [](float x, float y) { return x + y; };
    float top = 0.f, total = 0.f;
    if (!a.sigmoid && (group_value || !a.renorm)) {
        top = s[0];
#pragma unroll
        for (int r = 1; r < REGS; ++r) top = fmaxf(top, s[r]);
        top = over_lanes(top, LANES, most);
        top = top > none ? top : 0.f;
    }
    // v: p, then c; s itself where its order is asked for
    if (group_value || (!a.sigmoid && !a.renorm)) {
        float p[REGS];
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            if (a.sigmoid) p[r] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[r] * -1.4426950408889634f));
            else p[r] = __builtin_amdgcn_exp2f((s[r] - top) * 1.4426950408889634f);
        }
        if (!a.sigmoid) {
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < REGS; ++r) part[r & 3] += p[r];
            total = over_lanes((part[0] + part[1]) + (part[2] + part[3]), LANES, plus);
        }
        if (group_value) {
            const float by = a.sigmoid ? 1.0f : total > 0.f ? __builtin_amdgcn_rcpf(total) : 0.f;
#pragma unroll
            for (int r = 0; r < REGS; ++r) {
                const float c = by_value ? fmaf(p[r], by, v[r]) : p[r] * by;
                v[r] = s[r] > none ? c : none;
            }
        }
    }
    if (!group_value) {
#pragma unroll
        for (int r = 0; r < REGS; ++r) v[r] = s[r];
    }
    // two values that close may be in the other order: p is off by less than 2^-20, c by its own rounding too
    const auto close = [=](float x, float y) { return x > none && y > none && !(fabsf(x - y) > 0x1p-19f + 0x1p-22f * fmaxf(fabsf(x), fabsf(y))); };
    bool unsure = false, kept = true;
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
            unsure = unsure || (group_value && h != g && close(other, value));
        }
        kept = m1 > none && ahead < a.top_groups;
    }
    // without a bias experts are in the order of s
    double list[K];
    if constexpr (REGS <= K) {
#pragma unroll
        for (int r = 0; r < K; ++r) {
            const int m = first + r / VEC * (LG * VEC) + r % VEC;
            list[r] = r < REGS ? ranked(kept ? by_value ? v[r < REGS ? r : 0] : s[r < REGS ? r : 0] : none, g * S + m) : 0.0;
        }
        sort(list);
    } else {
#pragma unroll
        for (int b = 0; b < REGS; b += K) {
            double next[K];
#pragma unroll
            for (int r = 0; r < K; ++r) {
                const int m = first + (b + r) / VEC * (LG * VEC) + (b + r) % VEC;
                next[r] = ranked(kept ? by_value ? v[b + r] : s[b + r] : none, g * S + m);
            }
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

    // a slot per lane
    double mine = 0.0;
#pragma unroll
    for (int i = 0; i < K; ++i) mine = sub == i ? list[i] : mine;
    const bool full = sub < k && !ranked_none(mine);
    const int e = full ? ranked_expert(mine) : -1;
    float se = none;
    if (full) se = by_value ? read_score(a.bf16, static_cast<const char*>(a.scores) + row_at * (a.bf16 ? 2 : 4), e) : ranked_value(mine);
    if (by_value) {
        // an order hangs on neighbouring slots, unless they are alike, and on the last slot and every expert behind it
        const float value = full ? ranked_value(mine) : none, be = full ? a.bias[e] : 0.f;
        const int next = lane + 1;
        const float nv = __shfl(value, next, 64), ns = __shfl(se, next, 64), nb = __shfl(be, next, 64);
        const int ne = __shfl(e, next, 64);
        unsure = unsure || (sub + 1 < k && full && ne >= 0 && close(value, nv) && !(se == ns && be == nb));
        const int last = (lane & ~(LANES - 1)) + k - 1;
        const float lv = __shfl(value, last, 64);
        const int le = __shfl(e, last, 64);
        int found = 0;
#pragma unroll
        for (int r = 0; r < REGS; ++r) found += __popcll(__ballot(kept && le >= 0 && v[r] > none && (v[r] >= lv || close(v[r], lv))));
        if (found > __popcll(__ballot(full && le >= 0))) {   // of some token of the wavefront: look which, and at those that are like the last one
            const float ls = __shfl(se, last, 64), lb = __shfl(be, last, 64);
#pragma unroll
            for (int r = 0; r < REGS; ++r) {
                const int m = first + r / VEC * (LG * VEC) + r % VEC;
                if (kept && le >= 0 && v[r] > none && close(v[r], lv) && g * S + m != le) {
                    // chosen ones are close to the last slot only if a neighbour is: said above
                    const bool behind = v[r] < lv || (v[r] == lv && g * S + m > le);
                    unsure = unsure || (behind && !(s[r] == ls && a.bias[g * S + m] == lb));
                }
            }
        }
    }
    const Weights rule{a.sigmoid, a.renorm, a.scale};
    const float best_chosen = over_lanes(se, LANES, most);
    float w = slot_weight(rule, se, full, best_chosen, top, total);
    if (a.renorm) {
        const float sum = over_lanes(w, LANES, plus);
        w = sum > 0.f ? w / sum : 0.f;
    }
    unsigned long long again = __ballot(unsure && there);
    constexpr unsigned long long TOKEN = (1ull << LANES) - 1ull;
    if (there && sub < k && !((again >> (lane & ~(LANES - 1))) & TOKEN)) {
        a.idx[t * k + sub] = e;
        a.w[t * k + sub] = w * a.scale;
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
    hipLaunchKernelGGL((route_kernel<LANES, REGS, K, VEC>), dim3((unsigned)((a.T + tokens - 1) / tokens)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int LANES, int K, int VEC>
hipError_t launch_regs(const RouteArgs& a, int regs, hipStream_t s)
{
    if (regs <= 8) return launch<LANES, 8, K, VEC>(a, s);
    return regs <= 16 ? launch<LANES, 16, K, VEC>(a, s) : launch<LANES, 32, K, VEC>(a, s);
}

__global__ __launch_bounds__(256) void route_exact_kernel(RouteArgs a)
{
    __shared__ double s_c[4][kRtExperts];
    __shared__ int s_slot[4][kRtTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long t = (long long)blockIdx.x * 4 + wave;
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
        if (a.k <= 8 && a.groups <= 8 && regs(8) <= 32 && a.T > kRtFewTokens)
            return vec == 4 ? launch_regs<8, 8, 4>(a, regs(8), s) : launch_regs<8, 8, 1>(a, regs(8), s);
        if (regs(16) <= 32) {
            if (a.k <= 8) return vec == 4 ? launch_regs<16, 8, 4>(a, regs(16), s) : launch_regs<16, 8, 1>(a, regs(16), s);
            return vec == 4 ? launch_regs<16, 16, 4>(a, regs(16), s) : launch_regs<16, 16, 1>(a, regs(16), s);
        }
    }
    const dim3 grid((unsigned)(((long long)a.T + 3) / 4));
    hipLaunchKernelGGL(route_exact_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace moe_ep
