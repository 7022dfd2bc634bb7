// Norms behind and in front of a block, with the block's gate and the residual stream between them:
//   h = residual_scale residual + block_scale f(gate) N_after(block);   sum = h,  out = N_before(h)
// All of it is fp32 in registers, a row at a time: each operand is read once, each result rounded once and written once.  (Rows of more than 16384 elements with an operand in fp32
// have up to 105 registers a lane more than there are, in scratch memory: 1024 x 32768, block and stream in fp32, 138 us, 3.4 TB/s; in bf16, without, 63 us, 4.2 TB/s.)
#include <type_traits>

#include "rows.h"

namespace moe_ep {

namespace {

// 8 consecutive elements as they come from memory; WIDE: of either type, bf16 ones take the first half, else bf16
template <bool WIDE> struct Raw8 { u32x4_t v[WIDE ? 2 : 1]; };

// the `left` first of 8 elements, and zeros; cols: elements of the row
template <bool WIDE>
__device__ __forceinline__ Raw8<WIDE> load_raw(const char* row, int col, bool wide, int left, int cols)
{
    Raw8<WIDE> r;
    if constexpr (WIDE) {
        if (wide) {
            const float* const p = reinterpret_cast<const float*>(row) + col;
            r.v[0] = load_part<4>(p, left, cols);
            r.v[1] = load_part<4>(p + 4, left - 4, cols);
            return r;
        }
        r.v[1] = u32x4_t{0, 0, 0, 0};
    }
    r.v[0] = load_part<8>(reinterpret_cast<const uint16_t*>(row) + col, left, cols);
    return r;
}

template <bool WIDE>
__device__ __forceinline__ void to_float(const Raw8<WIDE>& r, bool wide, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float narrow = (i & 1) ? bf16_hi(r.v[0][i >> 1]) : bf16_lo(r.v[0][i >> 1]);
        if constexpr (WIDE) f[i] = wide ? __uint_as_float(r.v[i >> 2][i & 3]) : narrow;
        else f[i] = narrow;
    }
}

__device__ __forceinline__ void store8(char* row, int col, bool wide, int left, const float (&f)[8])
{
    if (left >= 8) {
        if (wide) {
            f32x4_any4* const p = reinterpret_cast<f32x4_any4*>(reinterpret_cast<float*>(row) + col);
            p[0] = f32x4_t{f[0], f[1], f[2], f[3]};
            p[1] = f32x4_t{f[4], f[5], f[6], f[7]};
        } else
            *reinterpret_cast<u32x4_any2*>(reinterpret_cast<uint16_t*>(row) + col) =
                u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        if (i >= left) continue;
        if (wide) reinterpret_cast<float*>(row)[col + i] = f[i];
        else reinterpret_cast<uint16_t*>(row)[col + i] = (uint16_t)pack_bf16x2(f[i], 0.f);
    }
}

struct Add { __device__ float operator()(float a, float b) const { return a + b; } };
struct Larger { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };   // of two numbers where one is NaN, the other

// over a wavefront's lanes, the same bits in every lane: as by exchanges of lanes 1, 2, 4, .. 32 apart, the mirrored ones of which hold what those would.  Without LDS (exchanges
// through it, us: 1531 x 1409, layer norms on both sides, 12.4 / 12.0, 4096 x 4096 38.6 / 34.6; RMS, 16384 x 5120, 120.8 / 119.1)
template <class Op>
__device__ __forceinline__ float over_wave(float v, Op op)
{
    const auto from = [&](auto control) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(control)::value, 0xf, 0xf, true)); };
    v = op(v, from(std::integral_constant<int, 0xb1>()));    // quad_perm 1 0 3 2
    v = op(v, from(std::integral_constant<int, 0x4e>()));    // quad_perm 2 3 0 1
    v = op(v, from(std::integral_constant<int, 0x141>()));   // row_half_mirror
    v = op(v, from(std::integral_constant<int, 0x140>()));   // row_mirror
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}

// N numbers over the WAVES wavefronts of a row, the same bits in every lane
constexpr int kOverRow = 2;
template <int WAVES, int N, class Op>
__device__ __forceinline__ void over_row(float (&v)[N], float* lds, int& turn, Op op)
{
    static_assert(N <= kOverRow, "norm_kernel's LDS");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = over_wave(v[i], op);
    if constexpr (WAVES > 1) {
        // two places in turn: who is at the next reduction has left this one's barrier, which everybody reaches behind reading the last one's
        float* const at = lds + (turn & 1) * (kOverRow * WAVES);
        ++turn;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) at[i * WAVES + (threadIdx.x >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = at[i * WAVES];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v[i] = op(v[i], at[i * WAVES + w]);
            if (N > 1) __builtin_amdgcn_sched_barrier(0);   // one number's sums after the other's: all at once are 2 WAVES registers
        }
    }
}

// x <- (x - mean) / sqrt(mean((x - mean)^2) + eps); RMS: without the mean.  The mean is taken out before the squares are summed, so that nothing cancels.
// What the mean is off by, a few steps of it, is all that is left of a row of equal numbers: the sum of what is left comes with that of its squares and is taken out too, and
// what the squares are of once more if it is a quarter of the result's unit or more.  So results are off by steps of their own, M / 64 + 20 at most, however large the mean is beside the spread.
// Where squares or sums leave fp32 while the row's numbers do not, its largest is between 2^56 (its square times 32768 is 2^127) and 2^128: times 2^-72 neither
// they nor anything that counts beside them is lost, and eps, which does not count there, goes with it, but to no less than a normal number: numbers that are all the
// mean have nothing else below the square root.  Such a row costs two or three reductions more.
constexpr float kScaled = 0x1p-72f;
__device__ __forceinline__ float scaled_eps(float eps) { return fmaxf(eps * kScaled * kScaled, __FLT_MIN__); }
template <int WAVES, int V>
__device__ __forceinline__ float largest(const float (&x)[V][8], float* lds, int& turn)
{
    float top[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) top[0] = fmaxf(top[0], fabsf(x[v][i]));
    over_row<WAVES>(top, lds, turn, Larger());
    return top[0];
}

template <int WAVES, int V>
__device__ __forceinline__ void normalise_rms(float (&x)[V][8], const int (&left)[V], int cols, float eps, float* lds, int& turn)
{
    const float each = 1.0f / (float)cols;
    for (int scaled = 0;; ++scaled) {
        float q[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < left[v] ? x[v][i] : 0.f;
                q[0] = fmaf(d, d, q[0]);
            }
        over_row<WAVES>(q, lds, turn, Add());
        const float power = q[0] * each;
        // (a number that is none, or infinite: as the formula has it)
        if (scaled == 0 && !(power <= __FLT_MAX__) && largest<WAVES, V>(x, lds, turn) <= __FLT_MAX__) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] *= kScaled;
            eps = scaled_eps(eps);
            continue;
        }
        const float r = __builtin_amdgcn_rsqf(power + eps);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] *= r;
        return;
    }
}

// Either kind.  The row stays as it is until the end: what a pass found out is in three numbers beside it.  (1531 x 1409, layer norms on both sides, without the sum of what is left /
// with it, us: 11.4 / 12.0.)
template <int WAVES, int V>
__device__ __forceinline__ void normalise_any(float (&x)[V][8], const int (&left)[V], int cols, bool layer, float eps, float* lds, int& turn)
{
#pragma clang fp contract(off)   // the same differences from the mean everywhere
    const float each = 1.0f / (float)cols;
    const auto mean_of = [&](float by) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] = fmaf(x[v][i], by, s[0]);
        over_row<WAVES>(s, lds, turn, Add());
        return s[0] * each;
    };
    float by = 1.f, mean = layer ? mean_of(1.f) : 0.f, rest = 0.f, last = 0.f, power = 0.f;
    const auto differ = [&](int v, int i) { return fmaf(x[v][i], by, -mean) - rest; };
    // a pass leaves 2^-15 of a mean or less: of 2^128 the ninth leaves less than a quarter of the root of the least eps
#pragma unroll 1
    for (int pass = 0; pass < 16; ++pass) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < left[v] ? differ(v, i) : 0.f;
                s[0] = fmaf(d, d, s[0]);
                s[1] += d;
            }
        over_row<WAVES>(s, lds, turn, Add());
        power = s[0] * each;
        if (by == 1.f && !(power <= __FLT_MAX__) && largest<WAVES, V>(x, lds, turn) <= __FLT_MAX__) {
            by = kScaled;
            eps = scaled_eps(eps);
            if (layer) mean = mean_of(by);
            continue;
        }
        if (!layer) break;
        last = s[1] * each;
        const float spread = fmaf(-last, last, power);
        power = spread < 0.f ? 0.f : spread;
        if (!(last * last > 0.0625f * (power + eps))) break;
        rest += last;
    }
    const float r = __builtin_amdgcn_rsqf(power + eps);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v][i] = (differ(v, i) - last) * r;
}

// LAYERS: it may be a layer norm
template <bool LAYERS, int WAVES, int V>
__device__ __forceinline__ void normalise(float (&x)[V][8], const int (&left)[V], int cols, int kind, float eps, float* lds, int& turn)
{
    if constexpr (LAYERS) normalise_any<WAVES, V>(x, left, cols, kind == kNormLayer, eps, lds, turn);
    else normalise_rms<WAVES, V>(x, left, cols, eps, lds, turn);
}

// A weight and a bias of 8 features
struct Weights { Raw8<true> weight, bias; };
__device__ __forceinline__ Weights load_weights(const NormArgs& a, const void* weight, const void* bias, int col, int left)
{
    Weights w;
    if (weight) w.weight = load_raw<true>(static_cast<const char*>(weight), col, a.weight32, left, a.M);
    if (bias) w.bias = load_raw<true>(static_cast<const char*>(bias), col, a.weight32, left, a.M);
    return w;
}
// x <- x (weight + offset) + bias
__device__ __forceinline__ void weigh(float (&x)[8], const NormArgs& a, const Weights& w, const void* weight, const void* bias)
{
    float f[8];
    if (weight) {
        to_float(w.weight, a.weight32, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= f[i] + a.offset;
    }
    if (bias) {
        to_float(w.bias, a.weight32, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += f[i];
    }
}

__device__ __forceinline__ float gate_of(float g, int form)
{
    if (form == kGateAsIs) return g;
    const float s = __builtin_amdgcn_rcpf(1.0f + exp_f(-g));
    return form == kGateSigmoid ? s : g * s;
}

// WAVES wavefronts have a row, a lane 8 elements of it in each of V turns.  WIDE: the block, the stream or the gate is fp32.  EARLY: weights and biases are asked for
// with the row, not behind the sums in front of them.  LAYERS: some norm is a layer norm, whose code costs others registers (RMS with it / without, us:
// 16384 x 5120 123 / 117, 4096 x 4096, norms on both sides, 32.5 / 30.2, 4096 x 32768 222 / 212).
// Of many rows memory bounds it: 16384 x 5120, bf16, residual and norm in front, 119 us for 671 MB, 5.6 TB/s (a copy of 1 GiB: 5.1); of few the chain of load, sum
// over wavefronts, square root, store: 1 x 5120 3.7 us, 4.5 with norms on both sides and nothing in L2.
template <int WAVES, int V, bool WIDE, bool EARLY, bool LAYERS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_kernel(NormArgs a)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float lds[2 * kOverRow * WAVES];
    int turn = 0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const long long m = workgroup() * ROWS + (WAVES == 1 ? wave : 0);
    if (m >= a.R) return;                                  // all of a row's wavefronts
    int col[V], left[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        col[v] = (v * WAVES * 64 + lane) * 8;
        left[v] = a.M - col[v];
        if (left[v] <= 0) { left[v] = 0; col[v] = 0; }
    }
    const char* const block = static_cast<const char*>(a.block) + (size_t)m * a.ldb * (a.block32 ? 4 : 2);
    const char* const residual = static_cast<const char*>(a.residual) + (size_t)m * a.ldr * (a.stream32 ? 4 : 2);
    const char* const gate = static_cast<const char*>(a.gate) + (size_t)m * a.ldg * (a.gate32 ? 4 : 2);

    Raw8<WIDE> b[V], r[V], g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) b[v] = load_raw<WIDE>(block, col[v], a.block32, left[v], a.M);
    if (a.residual)
#pragma unroll
        for (int v = 0; v < V; ++v) r[v] = load_raw<WIDE>(residual, col[v], a.stream32, left[v], a.M);
    const bool of_elements = a.gate && !a.gate_per_row;
    if (of_elements)
#pragma unroll
        for (int v = 0; v < V; ++v) g[v] = load_raw<WIDE>(gate, col[v], a.gate32, left[v], a.M);
    Weights after[V], before[V];
    if constexpr (EARLY)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            after[v] = load_weights(a, a.after_weight, a.after_bias, col[v], left[v]);
            before[v] = load_weights(a, a.before_weight, a.before_bias, col[v], left[v]);
        }
    float one = a.block_scale;
    if (a.gate && a.gate_per_row) one *= gate_of(a.gate32 ? *reinterpret_cast<const float*>(gate) : bf16_lo(*reinterpret_cast<const uint16_t*>(gate)), a.gate_form);

    float x[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) to_float(b[v], a.block32, x[v]);
    if (a.after != kNormNone) normalise<LAYERS, WAVES, V>(x, left, a.M, a.after, a.eps, lds, turn);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if constexpr (!EARLY) after[v] = load_weights(a, a.after_weight, a.after_bias, col[v], left[v]);
        weigh(x[v], a, after[v], a.after_weight, a.after_bias);
    }
    if (of_elements)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float f[8];
            to_float(g[v], a.gate32, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] *= gate_of(f[i], a.gate_form);
        }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float f[8];
        if (a.residual) to_float(r[v], a.stream32, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v][i] = a.residual ? fmaf(a.residual_scale, f[i], one * x[v][i]) : one * x[v][i];
    }
    if (a.sum) {
        char* const sum = static_cast<char*>(a.sum) + (size_t)m * a.lds * (a.stream32 ? 4 : 2);
#pragma unroll
        for (int v = 0; v < V; ++v) store8(sum, col[v], a.stream32, left[v], x[v]);
    }
    if (!a.out) return;
    // what is not there counts as zero
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v][i] = i < left[v] ? x[v][i] : 0.f;
    normalise<LAYERS, WAVES, V>(x, left, a.M, a.before, a.eps, lds, turn);
    char* const out = static_cast<char*>(a.out) + (size_t)m * a.ldo * (a.out32 ? 4 : 2);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if constexpr (!EARLY) before[v] = load_weights(a, a.before_weight, a.before_bias, col[v], left[v]);
        weigh(x[v], a, before[v], a.before_weight, a.before_bias);
        store8(out, col[v], a.out32, left[v], x[v]);
    }
}

template <int WAVES, int V, bool EARLY>
hipError_t launch_as(const NormArgs& a, hipStream_t s)
{
    const long long groups = WAVES == 1 ? ((long long)a.R + 3) / 4 : a.R;
    const dim3 threads(WAVES == 1 ? 256 : WAVES * 64);
    const bool wide = a.block32 || a.stream32 || (a.gate32 && !a.gate_per_row);
    const auto launch = [&](auto layers) {
        if (wide) hipLaunchKernelGGL((norm_kernel<WAVES, V, true, EARLY, decltype(layers)::value>), grid_of(groups), threads, 0, s, a);
        else hipLaunchKernelGGL((norm_kernel<WAVES, V, false, EARLY, decltype(layers)::value>), grid_of(groups), threads, 0, s, a);
    };
    if (a.after == kNormLayer || a.before == kNormLayer) launch(std::true_type{}); else launch(std::false_type{});
    return hipGetLastError();
}

template <int WAVES, int V>
hipError_t launch_when(bool early, const NormArgs& a, hipStream_t s) { return early ? launch_as<WAVES, V, true>(a, s) : launch_as<WAVES, V, false>(a, s); }

}  // namespace

// The least that holds a row, in one turn up to 4096 elements.  Residual and norm of bf16 rows, turns x wavefronts, us: 1 / 1024 / 16384 x 2048 1 x 4 2.9 / 6.0 /
// 48, 2 x 2 3.3 / 6.2 / 47, 4 x 1 5.5 / 8.4 / 52; x 4096 1 x 8 3.1 / 9.0 / 98, 2 x 4 3.4 / 8.9 / 96, 4 x 2 5.3 / 11 / 99.  Beyond 4096 the turns are two where compute units have
// several rows: 1 x 16 / 2 x 8, of norms on both sides, operands not in L2, 1, 33, 256, 512 x 5120 4.5 / 4.6, 5.2 / 5.6, 6.4 / 6.9, 11 / 10, 256 x 8192 7.8 / 7.8; of one norm, 1024, 16384
// x 5120 14 / 11, 170 / 119.
int norm_kernel_of(int R, int M, int n_cu)
{
    if (M > 4096 && M <= 8192) return R <= n_cu ? kNorm16x1 : kNorm8x2;
    return M <= 512 ? kNorm1x1 : M <= 1024 ? kNorm2x1 : M <= 2048 ? kNorm4x1 : M <= 4096 ? kNorm8x1 : M <= 16384 ? kNorm16x2 : kNorm16x4;
}

hipError_t launch_norm(const NormArgs& a, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.M < 1 || a.M > kNormMost) return hipErrorInvalidValue;
    // With a row for every compute unit, or fewer, nothing but the row's own loads hides those of the weights.  Weights asked for behind the sums / with the row, norms on
    // both sides, operands not in L2, us: 1, 33, 256, 512 x 2048 3.6 / 3.1, 4.1 / 3.5, 5.1 / 4.3, 5.7 / 5.3; x 4096 4.0 / 3.4, 5.2 / 4.3, 6.0 / 5.3, 7.7 / 7.4.  With more rows the registers
    // that they take are wavefronts less: of an RMS norm in front that costs least (16384 x 2048, 4096 50 / 48, 101 / 94, norms on both sides 55 / 56, 125 / 107, a gate an element 66 / 68,
    // 149 / 127), of layer norms it is as often worse (49 / 52, 104 / 103, on both sides 73 / 73, 161 / 147, 4096 rows 24 / 24, 43 / 43), without a norm in front it is (38 / 39, 69 / 71).
    const bool early = a.R <= n_cu || (a.before == kNormRms && a.after != kNormLayer);
    switch (norm_kernel_of(a.R, a.M, n_cu)) {
    case kNorm1x1: return launch_when<1, 1>(early, a, s);
    case kNorm2x1: return launch_when<2, 1>(early, a, s);
    case kNorm4x1: return launch_when<4, 1>(early, a, s);
    case kNorm8x1: return launch_when<8, 1>(early, a, s);
    case kNorm16x1: return launch_as<16, 1, true>(a, s);
    case kNorm8x2: return launch_as<8, 2, false>(a, s);
    case kNorm16x2: return launch_as<16, 2, false>(a, s);
    default: return launch_as<16, 4, false>(a, s);
    }
}

}  // namespace moe_ep
