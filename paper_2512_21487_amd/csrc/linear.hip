// Matrix product with an epilogue: out = act(x W^T + bias) + residual, for the gate's scores (weights in fp32) and for dense layers.
// Both operands are K-contiguous, which is what the bf16 matrix instructions want per lane; the weight rows are the first operand, so
// that a lane ends up with four consecutive output columns of one row.  Sums, bias, activation and residual are fp32; a result is
// rounded once.
//
// fp32 weights are three bf16 numbers each, 8 mantissa bits at a time cut off the top (24 together: all of them), and a product is three
// matrix instructions: as exact as fp32 multiplications at 5 times their rate.
#include <atomic>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace moe_ep {

namespace {

#define SB() __builtin_amdgcn_sched_barrier(0)

// 16 or 8 bytes from an address that only the type of the elements aligns
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// exp from the hardware's exp2: off by about a step of fp32 and by what the argument's own rounding makes of it
__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// 0.5 z (1 + erf(z / sqrt 2)).  1 - erf(x) for x >= 0 is a polynomial in 1 / (1 + p x) times exp(-x^2) to 1.5e-7 (Abramowitz and Stegun,
// Handbook of Mathematical Functions, 7.1.26), so that nothing cancels where z is negative.  Of z from N(0, 1) it is off by 8.4e-8 (RMS, of the result's)
// and 3.3e-7 at most, the formula in fp32 by 3.8e-8 and 3.8e-7; half a step of bf16 is 3.9e-3, and sums of a few products are off by more.
__device__ __forceinline__ float gelu_f(float z)
{
    const float x = fabsf(z) * 0.7071067811865476f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float h = 0.5f * fminf(z, __FLT_MAX__) * (q * exp_f(-x * x));   // 0.5 z (1 - erf(x)), 0 of plus infinity
    return z >= 0.f ? z - h : h;
}

// 0.5 z (1 + tanh(u)) = z / (1 + exp(-2u)),  u = sqrt(2 / pi) (z + 0.044715 z^3)
__device__ __forceinline__ float gelu_tanh_f(float z)
{
    const float u = 0.7978845608028654f * (z + 0.044715f * z * z * z);
    return z * __builtin_amdgcn_rcpf(1.0f + exp_f(-2.0f * u));
}

// one branch for N numbers
template <int N, class V>
__device__ __forceinline__ void activate(int act, V& v)
{
    switch (act) {
    case kActRelu:
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];   // a NaN stays one
        break;
    case kActSilu:
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = silu_f(v[i]);
        break;
    case kActGelu:
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gelu_f(v[i]);
        break;
    case kActGeluTanh:
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gelu_tanh_f(v[i]);
        break;
    default: break;
    }
}

// Epilogue of 16 rows x NB * 16 columns in registers: a lane has 4 consecutive columns of its row in every block of 16.
template <int NB>
struct Epilogue {
    struct Residual { u32x4_t v[NB]; };          // bf16 ones take the first half
    const LinearArgs& a;
    int n, kh;                                   // the lane's column in block 0; which four of the block's 16 columns
    bool whole;                                  // every column of the wavefront is there
    f32x4_t bias[NB];

    __device__ __forceinline__ Epilogue(const LinearArgs& args, int n0, int kh_) : a(args), n(n0 + kh_ * 4), kh(kh_), whole(n0 + NB * 16 <= args.N)
    {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            bias[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (!a.bias) continue;
            if (whole) bias[b] = *reinterpret_cast<const f32x4_any4*>(a.bias + n + b * 16);
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) bias[b][i] = a.bias[min(n + b * 16 + i, a.N - 1)];
        }
    }
    __device__ __forceinline__ bool group(int b) const { return whole || n + b * 16 + 4 <= a.N; }   // all four columns in block b
    // of a row that is there
    __device__ __forceinline__ void fetch(int m, Residual& r) const
    {
        const char* const row = static_cast<const char*>(a.residual) + ((size_t)m * a.ldr + n) * (a.out32 ? 4 : 2);
        if (a.out32) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
                if (group(b)) r.v[b] = *reinterpret_cast<const u32x4_any2*>(row + b * 64);
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
                if (group(b)) {
                    const u32x2_t x = *reinterpret_cast<const u32x2_any2*>(row + b * 32);
                    r.v[b] = u32x4_t{x[0], x[1], 0, 0};
                }
        }
    }
    __device__ __forceinline__ void store(int m, bool there, f32x4_t v[NB], const Residual& res) const
    {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v[b] += bias[b];
            activate<4>(a.act, v[b]);
        }
        if (a.residual) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (!group(b)) continue;
                const u32x4_t r = res.v[b];
                v[b] += a.out32 ? __builtin_bit_cast(f32x4_t, r) : f32x4_t{bf16_lo(r[0]), bf16_hi(r[0]), bf16_lo(r[1]), bf16_hi(r[1])};
            }
        }
        char* const row = static_cast<char*>(a.out) + ((size_t)m * a.ldo + n) * (a.out32 ? 4 : 2);
        if (whole && !a.out32) {
            // two neighbouring blocks exchange halves: 8 columns of one of them a lane, 64 bytes of a row a store
            char* const at = row + ((kh & 1) * 16 + (kh >> 1) * 8 - kh * 4) * 2;
#pragma unroll
            for (int b = 0; b + 1 < NB; b += 2) {
                const f32x4_t u = v[b], w = v[b + 1];
                const auto s0 = __builtin_amdgcn_permlane16_swap(pack_bf16x2(u[0], u[1]), pack_bf16x2(w[0], w[1]), false, false);
                const auto s1 = __builtin_amdgcn_permlane16_swap(pack_bf16x2(u[2], u[3]), pack_bf16x2(w[2], w[3]), false, false);
                if (there) *reinterpret_cast<u32x4_any2*>(at + b * 32) = u32x4_t{s0[0], s1[0], s0[1], s1[1]};
            }
        }
        if (!there) return;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (whole && !a.out32 && !(NB % 2 && b == NB - 1)) continue;
            if (!group(b)) continue;
            if (a.out32) *reinterpret_cast<f32x4_any4*>(row + b * 64) = v[b];
            else *reinterpret_cast<u32x2_any2*>(row + b * 32) = u32x2_t{pack_bf16x2(v[b][0], v[b][1]), pack_bf16x2(v[b][2], v[b][3])};
        }
        if (whole || a.N % 4 == 0) return;
        // the last columns, fewer than four, of whichever block they are in
        const int left = a.N - n, last = left >> 4;
        if (left < 0 || (left & 15) > 3 || last >= NB) return;
        f32x4_t u = v[0];
#pragma unroll
        for (int b = 1; b < NB; ++b) u = last == b ? v[b] : u;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (i >= (left & 15)) continue;
            const size_t from = (size_t)m * a.ldr + n + last * 16 + i;
            float x = u[i];
            if (a.out32) reinterpret_cast<float*>(row)[last * 16 + i] = a.residual ? x + static_cast<const float*>(a.residual)[from] : x;
            else reinterpret_cast<uint16_t*>(row)[last * 16 + i] = (uint16_t)pack_bf16x2(a.residual ? x + bf16_lo(static_cast<const uint16_t*>(a.residual)[from]) : x, 0.f);
        }
    }
};

// 8 elements of a row, the `left` first of which are there, and zeros; p: the first
__device__ __forceinline__ u32x4_t load8(const uint16_t* p, int left)
{
    if (left >= 8) return *reinterpret_cast<const u32x4_any2*>(p);
    u32x4_t v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i) if (i < left) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    return v;
}
struct f32x8_t { f32x4_t lo, hi; };
__device__ __forceinline__ f32x8_t load8(const float* p, int left)
{
    f32x8_t v;
    if (left >= 8) {
        v.lo = *reinterpret_cast<const f32x4_any4*>(p);
        v.hi = *reinterpret_cast<const f32x4_any4*>(p + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v.lo[i] = i < left ? p[i] : 0.f; v.hi[i] = i + 4 < left ? p[i + 4] : 0.f; }
    }
    return v;
}

// 16 bytes of a row, the `left` first elements of which are there, and zeros.  A row of N elements and more: its last 16 bytes, shifted
// (an element at a time, the last K step of 1531 x 1409 x 2049 took 7 of 49 us).
template <int N, class T>
__device__ __forceinline__ u32x4_t load_part(const T* p, int left, int cols)
{
    if (left >= N) return *reinterpret_cast<const u32x4_any2*>(p);
    u32x4_t v = {0, 0, 0, 0};
    if (cols >= N) {
        if (left <= 0) return v;
        const u32x4_t u = *reinterpret_cast<const u32x4_any2*>(p - (N - left));
        const uint64_t lo = (uint64_t)u[1] << 32 | u[0], hi = (uint64_t)u[3] << 32 | u[2];
        const int drop = (N - left) * (128 / N);                     // bits, 16 .. 112
        const uint64_t a = drop < 64 ? lo >> drop | hi << (64 - drop) : hi >> (drop - 64), b = drop < 64 ? hi >> drop : 0;
        return u32x4_t{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        if (i >= left) continue;
        if constexpr (N == 8) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        else v[i] = __float_as_uint(p[i]);
    }
    return v;
}

// The kernel may ask for `bytes` of LDS: told once per device, of the first 64
template <class K>
hipError_t allow_lds(K* kernel, int bytes, std::atomic<uint64_t>& told)
{
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess || (device < 64 && (told.load(std::memory_order_relaxed) >> device & 1))) return e;
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && device < 64) told.fetch_or(1ull << device, std::memory_order_relaxed);
    return e;
}

// ---- a few rows: no matrix instruction is full

// A workgroup has C columns and up to RB rows: its threads take 8 elements of the reduction in turn, which reads the weights in whole
// 4 or 8 KB, and their sums are added up through the wavefronts and LDS.  Latency bounds it: 1 x 160 x 5120 with fp32 weights 3.1 us (with 16
// rows of a matrix instruction, 15 of them empty, 8.6), of which reading 3.3 MB is 0.6.
template <int RB, int C, bool W32>
__global__ __launch_bounds__(256) void linear_rows_kernel(LinearArgs a)
{
    __shared__ float s_sum[4][C * RB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nt = (a.N + C - 1) / C, n0 = (int)(blockIdx.x % nt) * C, m0 = (int)(blockIdx.x / nt) * RB;
    float acc[C][RB];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[c][r] = 0.f;
    typedef typename std::conditional<W32, float, uint16_t>::type Weight;
    typedef typename std::conditional<W32, f32x8_t, u32x4_t>::type Weight8;
#pragma unroll 2
    for (int k = tid * 8; k < a.K; k += 256 * 8) {
        const int left = a.K - k;
        Weight8 w[C];
        u32x4_t x[RB];
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = load8(static_cast<const Weight*>(a.w) + (size_t)min(n0 + c, a.N - 1) * a.ldw + k, left);
#pragma unroll
        for (int r = 0; r < RB; ++r) x[r] = load8(a.x + (size_t)min(m0 + r, a.R - 1) * a.ldx + k, left);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (W32) f[i] = i < 4 ? w[c].lo[i & 3] : w[c].hi[i & 3];
                else f[i] = (i & 1) ? bf16_hi(w[c][i >> 1]) : bf16_lo(w[c][i >> 1]);
            }
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[c][r] = fmaf(f[i], (i & 1) ? bf16_hi(x[r][i >> 1]) : bf16_lo(x[r][i >> 1]), acc[c][r]);
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float v = acc[c][r];
#pragma unroll
            for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
            if (lane == 0) s_sum[wave][r * C + c] = v;
        }
    __syncthreads();
    if (tid < C * RB) {
        const int m = m0 + tid / C, n = n0 + tid % C;
        if (m < a.R && n < a.N) {
            float v[1] = {s_sum[0][tid] + s_sum[1][tid] + s_sum[2][tid] + s_sum[3][tid]};
            if (a.bias) v[0] += a.bias[n];
            activate<1>(a.act, v);
            const size_t from = (size_t)m * a.ldr + n, to = (size_t)m * a.ldo + n;
            if (a.residual) v[0] += a.out32 ? static_cast<const float*>(a.residual)[from] : bf16_lo(static_cast<const uint16_t*>(a.residual)[from]);
            if (a.out32) static_cast<float*>(a.out)[to] = v[0];
            else static_cast<uint16_t*>(a.out)[to] = (uint16_t)pack_bf16x2(v[0], 0.f);
        }
    }
}

template <int RB, int C>
hipError_t launch_rows(const LinearArgs& a, hipStream_t s)
{
    const long long grid = (long long)((a.N + C - 1) / C) * ((a.R + RB - 1) / RB);
    if (grid > 0x7fffffffll) return hipErrorInvalidValue;
    if (a.w32) hipLaunchKernelGGL((linear_rows_kernel<RB, C, true>), dim3((unsigned)grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((linear_rows_kernel<RB, C, false>), dim3((unsigned)grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

// ---- some rows, weights in fp32, or operands that are not on 16 bytes

// the upper halves of two words, of `a` in the low half
__device__ __forceinline__ uint32_t upper_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }

// 8 fp32 numbers as the sum of three times 8 bf16 numbers
__device__ __forceinline__ void split3(const f32x8_t& w, bf16x8_t part[3])
{
    float r[8] = {w.lo[0], w.lo[1], w.lo[2], w.lo[3], w.hi[0], w.hi[1], w.hi[2], w.hi[3]};
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        const u32x4_t u = {upper_halves(r[0], r[1]), upper_halves(r[2], r[3]), upper_halves(r[4], r[5]), upper_halves(r[6], r[7])};
        part[j] = __builtin_bit_cast(bf16x8_t, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] -= __uint_as_float(__float_as_uint(r[i]) & 0xffff0000u);
    }
}

// The wavefronts of a workgroup share a tile of MB x NB blocks of 16 rows x 16 columns and take K steps of 64 of it in turn; their sums are added up
// in LDS, in the order of the wavefronts.  A step's rows are fetched in whole pieces of 128 or 256 bytes, at any alignment, and go through LDS of
// the wavefront's own (16-byte chunks XOR-swizzled by the row) to the lanes that multiply them, while the next step's are on their way.  Straight into
// those lanes, 16 rows' bytes at a time, a load took the memory path four times as long (4096 x 128 x 4096, fp32 weights: 33 us against 22).
// Those 22 us are 1.6 TB/s of operands; the matrix unit is busy 16 % of them.  What bounds it is a step's chain in each wavefront, LDS write, read,
// cutting the weights up, products, with only two wavefronts per SIMD to fill one another's gaps (eight slices of 16 KB are most of the LDS).
template <int MB, int NB, bool W32>
struct SplitCfg {
    static constexpr int KS = 64, WROW = W32 ? 256 : 128;                    // bytes of a row of weights
    static constexpr int XL = MB * 2, WL = NB * 16 * WROW / 1024;             // loads of 1 KB
    static constexpr int X_BYTES = MB * 16 * 128, W_BYTES = NB * 16 * WROW, BYTES = X_BYTES + W_BYTES;
    static_assert(MB * NB * 1024 <= BYTES, "the sums take the place of the operands");
};

template <int MB, int NB, int WAVES, bool W32>
__global__ __launch_bounds__(WAVES * 64) void linear_split_kernel(LinearArgs a)
{
    using C = SplitCfg<MB, NB, W32>;
    constexpr int KS = C::KS;
    extern __shared__ uint4 lds4[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* const own = reinterpret_cast<char*>(lds4) + wave * C::BYTES;
    // tiles of one XCD (workgroup number mod 8) are consecutive ones
    const int mt = (a.R + MB * 16 - 1) / (MB * 16), nt = (a.N + NB * 16 - 1) / (NB * 16);
    const long long total = (long long)mt * nt, per = (total + 7) / 8, at = workgroup(), L = (at & 7) * per + (at >> 3);
    if ((at >> 3) >= per || L >= total) return;
    const int m0 = (int)(a.rows_first ? L % mt : L / nt) * (MB * 16), n0 = (int)(a.rows_first ? L / mt : L % nt) * (NB * 16);

    // load i of the rows: 8 of x, or of bf16 weights, 8 lanes each; 4 of fp32 weights, 16 lanes each
    typedef typename std::conditional<W32, float, uint16_t>::type Weight;
    constexpr int PER = W32 ? 4 : 8;                                          // weights in 16 bytes
    const int xr = lane >> 3, xc = lane & 7, wr = W32 ? lane >> 4 : lane >> 3, wc = W32 ? lane & 15 : lane & 7;
    const uint16_t* const x0 = a.x + (size_t)m0 * a.ldx;
    const Weight* const w0 = static_cast<const Weight*>(a.w) + (size_t)n0 * a.ldw;
    // a tile's rows from its first: 64 rows of 2^22 elements are within 32 bits
    uint32_t xo[C::XL], wo[C::WL];
#pragma unroll
    for (int i = 0; i < C::XL; ++i) xo[i] = (uint32_t)min(i * 8 + xr, a.R - 1 - m0) * (uint32_t)a.ldx + xc * 8;
#pragma unroll
    for (int i = 0; i < C::WL; ++i) wo[i] = (uint32_t)min(i * (64 / (C::WROW / 16)) + wr, a.N - 1 - n0) * (uint32_t)a.ldw + wc * PER;
    struct Step { u32x4_t x[C::XL], w[C::WL]; } f;
    // whole: all 64 elements are there
    const auto load = [&](int step, bool whole) __attribute__((always_inline)) {
        const int left = a.K - step * KS;
#pragma unroll
        for (int i = 0; i < C::WL; ++i) {
            const Weight* p = w0 + step * KS + wo[i];
            f.w[i] = whole ? *reinterpret_cast<const u32x4_any2*>(p) : load_part<PER>(p, left - wc * PER, a.K);
        }
#pragma unroll
        for (int i = 0; i < C::XL; ++i) {
            const uint16_t* p = x0 + step * KS + xo[i];
            f.x[i] = whole ? *reinterpret_cast<const u32x4_any2*>(p) : load_part<8>(p, left - xc * 8, a.K);
        }
    };
    const uint32_t xw = xr * 128, ww = C::X_BYTES + wr * C::WROW;
    const auto to_lds = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C::WL; ++i) {
            const int r = i * (64 / (C::WROW / 16)) + wr, sw = W32 ? r & 15 : (r >> 1) & 7;
            *reinterpret_cast<u32x4_t*>(own + ww + i * 1024 + (wc ^ sw) * 16) = f.w[i];
        }
#pragma unroll
        for (int i = 0; i < C::XL; ++i) *reinterpret_cast<u32x4_t*>(own + xw + i * 1024 + (xc ^ (((i * 8 + xr) >> 1) & 7)) * 16) = f.x[i];
    };

    const int row = lane & 15, kh = lane >> 4, sw = (row >> 1) & 7, sw32 = row;
    f32x4_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const auto multiply = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8_t x[MB];
#pragma unroll
            for (int i = 0; i < MB; ++i) x[i] = *reinterpret_cast<const bf16x8_t*>(own + (i * 16 + row) * 128 + ((h * 4 + kh) ^ sw) * 16);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const char* const at = own + C::X_BYTES + (j * 16 + row) * C::WROW;
                if constexpr (W32) {
                    f32x8_t v;
                    v.lo = *reinterpret_cast<const f32x4_t*>(at + ((h * 8 + kh * 2) ^ sw32) * 16);
                    v.hi = *reinterpret_cast<const f32x4_t*>(at + ((h * 8 + kh * 2 + 1) ^ sw32) * 16);
                    bf16x8_t part[3];
                    split3(v, part);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
#pragma unroll
                        for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[p], x[i], acc[i][j], 0, 0, 0);
                } else {
                    const bf16x8_t w = *reinterpret_cast<const bf16x8_t*>(at + ((h * 4 + kh) ^ sw) * 16);
#pragma unroll
                    for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[i], acc[i][j], 0, 0, 0);
                }
            }
        }
    };
    const int steps = (a.K + KS - 1) / KS, whole = a.K / KS;
    if (wave < steps) load(wave, wave < whole);
    for (int st = wave; st < steps; st += WAVES) {
        to_lds();
        wavefront_lds_order();
        if (st + WAVES < steps) load(st + WAVES, st + WAVES < whole);
        SB();   // or the compiler moves loads behind the products
        multiply();
        wavefront_lds_order();
    }
    // a wavefront's operands make room for its sums
    f32x4_t* const sums = reinterpret_cast<f32x4_t*>(own) + lane;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[(i * NB + j) * 64] = acc[i][j];
    __syncthreads();
    // 16 rows a wavefront
    for (int i = wave; i < MB; i += WAVES) {
        const Epilogue<NB> e(a, n0, kh);
        const int m = m0 + i * 16 + row;
        typename Epilogue<NB>::Residual res;
        if (a.residual && m < a.R) e.fetch(m, res);
        f32x4_t v[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const f32x4_t* const at = reinterpret_cast<const f32x4_t*>(lds4) + (i * NB + j) * 64 + lane;
            v[j] = at[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v[j] += at[w * (C::BYTES / 16)];
        }
        e.store(m, m < a.R, v, res);
    }
}

template <int MB, int NB, int WAVES, bool W32>
hipError_t launch_split_as(const LinearArgs& a, long long workgroups, hipStream_t s)
{
    constexpr int bytes = WAVES * SplitCfg<MB, NB, W32>::BYTES;
    static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> told{0};
    const hipError_t e = allow_lds(&linear_split_kernel<MB, NB, WAVES, W32>, bytes, told);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((linear_split_kernel<MB, NB, WAVES, W32>), grid_of(workgroups), dim3(WAVES * 64), bytes, s, a);
    return hipGetLastError();
}

template <int MB, int NB, int WAVES>
hipError_t launch_split(LinearArgs a, hipStream_t s)
{
    const long long mt = (a.R + MB * 16 - 1) / (MB * 16), nt = (a.N + NB * 16 - 1) / (NB * 16), per = (mt * nt + 7) / 8;
    // an XCD's tiles share the rows of the larger operand through its L2
    a.rows_first = (double)a.N * a.K * (a.w32 ? 4 : 2) > (double)a.R * a.K * 2;
    return a.w32 ? launch_split_as<MB, NB, WAVES, true>(a, per * 8, s) : launch_split_as<MB, NB, WAVES, false>(a, per * 8, s);
}

// ---- many rows and columns


// 16 bytes per lane from memory to consecutive places in LDS.  Written out because the compiler cannot tell which slot a load is on its way to, and
// makes a fragment read in the middle of a K step wait for all of them; hand_over() is what waits.
__device__ __forceinline__ void load_to_lds(uint32_t to, const char* base, uint32_t off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(uint32_t to, const char* src)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src) : "memory", "m0");
}

__device__ const uint4 kZeros[4] = {};   // what a lane fetches that is beyond its row's end

// Many rows and columns: tiles of BM rows x BN columns through LDS, 2 x 2 wavefronts.  A K step is 64 elements, rows of 128 bytes
// whose 16-byte chunks are XOR-swizzled by the row, so that fragment reads meet no bank twice; global_load_lds brings them in, into a ring of
// SLOTS K steps.  A workgroup takes tiles in turn; the loads run ahead of the multiplications across tiles too.
template <int BM, int BN, int SLOTS>
struct TileCfg {
    static constexpr int KS = 64, NW = 4;
    static constexpr int WTM = BM / 2, WTN = BN / 2, MB = WTM / 16, NB = WTN / 16;
    static constexpr int RX = BM / 8 / NW, RW = BN / 8 / NW, RPW = RX + RW;   // 1 KB regions (8 rows) a wavefront loads per K step
    static constexpr int SLOT_BYTES = (BM + BN) * KS * 2;
    static constexpr int SUM_BYTES = 16 * WTN * 4;                            // epilogue: a wavefront's row of blocks in fp32
    static constexpr int LDS_BYTES = SLOTS * SLOT_BYTES + NW * SUM_BYTES;
    static constexpr int M = 2 * MB * NB;                                     // MFMAs of a K step
    static constexpr int TAIL = M / 4 > MB + NB ? M / 4 : MB + NB;            // of which behind the hand-over of the next slot
    static constexpr int HO = M - TAIL, WINDOW = M * 3 / 4 > RPW ? M * 3 / 4 : RPW;
    static constexpr int RD = 2 * (MB + NB) <= MB * NB ? 2 : 1;               // MFMAs between two fragment reads
    static_assert(MB + NB <= MB * NB && TAIL <= MB * NB, "reads of a step of 32 fit behind its MFMAs");
    // the load issued behind MFMA p after a hand-over, or -1
    static constexpr int load_at(int p)
    {
        const int l = (p * RPW + WINDOW - 1) / WINDOW;
        return l < RPW && l * WINDOW / RPW == p ? l : -1;
    }
};

// Epilogue of a wavefront's part of a tile, MB * 16 rows x COLS columns.  Bias and activation are applied where the sums are, a row of blocks at a
// time; that goes through LDS (fp32, 16-byte chunks XOR-swizzled by the row), so that residual and results move in whole pieces of a row: a lane has 8
// consecutive columns of every (64 / LANES)th row.  Straight from the accumulators, 8 bytes of 16 rows at a time, the residual alone took
// 80 us of 16384 x 5120 x 5120 instead of 8.
template <int MB, int COLS, bool ACT>
struct TileEpilogue {
    static constexpr int NB = COLS / 16, LANES = COLS > 64 ? 16 : COLS > 32 ? 8 : 4, ROWS = 64 / LANES, PASSES = 16 / ROWS;
    static_assert(COLS % 32 == 0 && COLS <= 128, "rows of whole swizzled groups of chunks");
    struct Residual { u32x4_t v[PASSES][2]; };   // 8 numbers; bf16 ones take the first half

    const LinearArgs& a;
    char* sums;
    const char* res_at;                          // of the wavefront's first row and column; a lane adds 32 bits (256 rows of 2^22 numbers fit)
    char* out_at;
    int rows, left, r0;                          // rows that are there; columns that are, from the lane's first; the lane's row in a pass
    uint32_t res_off, out_off, write, read;
    f32x4_t bias[NB];

    // m, n: the wavefront's first row and column
    __device__ __forceinline__ TileEpilogue(const LinearArgs& args, char* lds, int lane, int m, int n) : a(args), sums(lds), rows(args.R - m)
    {
        const int size = a.out32 ? 4 : 2, c = min(lane % LANES, COLS / 8 - 1), fr = lane & 15, kh = lane >> 4;
        r0 = lane / LANES;
        left = c == lane % LANES ? a.N - n - c * 8 : 0;
        res_at = static_cast<const char*>(a.residual) + ((size_t)m * a.ldr + n) * size;
        out_at = static_cast<char*>(a.out) + ((size_t)m * a.ldo + n) * size;
        res_off = (uint32_t)(r0 * (uint32_t)a.ldr + c * 8) * size;
        out_off = (uint32_t)(r0 * (uint32_t)a.ldo + c * 8) * size;
        write = fr * (COLS * 4) + ((kh ^ (fr & 3)) + (fr & 4)) * 16;
        read = r0 * (COLS * 4) + ((2 * c) ^ (r0 & 7)) * 16;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) bias[b][i] = a.bias ? a.bias[min(n + b * 16 + kh * 4 + i, a.N - 1)] : 0.f;
    }
    __device__ __forceinline__ bool there(int mb, int p) const { return mb * 16 + p * ROWS + r0 < rows; }
    __device__ __forceinline__ void fetch(int mb, Residual& r) const
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            if (!there(mb, p) || left < 8) continue;
            const char* const at = res_at + (res_off + (uint32_t)(mb * 16 + p * ROWS) * (uint32_t)a.ldr * (a.out32 ? 4u : 2u));
            r.v[p][0] = *reinterpret_cast<const u32x4_any2*>(at);
            if (a.out32) r.v[p][1] = *reinterpret_cast<const u32x4_any2*>(at + 16);
        }
    }
    __device__ __forceinline__ void store(int mb, f32x4_t (&v)[NB], const Residual& res) const
    {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v[b] += bias[b];
            if (ACT) activate<4>(a.act, v[b]);
            *reinterpret_cast<f32x4_t*>(sums + (b % 2 ? write ^ 64u : write) + b / 2 * 128) = v[b];
        }
        wavefront_lds_order();
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const uint32_t from = (read ^ (p * ROWS & 7) * 16) + p * ROWS * COLS * 4;
            f32x4_t lo = *reinterpret_cast<const f32x4_t*>(sums + from), hi = *reinterpret_cast<const f32x4_t*>(sums + (from ^ 16u));
            if (!there(mb, p) || left < 8) continue;
            if (a.residual) {
                const u32x4_t r = res.v[p][0];
                if (a.out32) {
                    lo += __builtin_bit_cast(f32x4_t, r);
                    hi += __builtin_bit_cast(f32x4_t, res.v[p][1]);
                } else {
                    lo += f32x4_t{bf16_lo(r[0]), bf16_hi(r[0]), bf16_lo(r[1]), bf16_hi(r[1])};
                    hi += f32x4_t{bf16_lo(r[2]), bf16_hi(r[2]), bf16_lo(r[3]), bf16_hi(r[3])};
                }
            }
            char* const to = out_at + (out_off + (uint32_t)(mb * 16 + p * ROWS) * (uint32_t)a.ldo * (a.out32 ? 4u : 2u));
            if (a.out32) {
                *reinterpret_cast<f32x4_any4*>(to) = lo;
                *reinterpret_cast<f32x4_any4*>(to + 16) = hi;
            } else *reinterpret_cast<u32x4_any2*>(to) = u32x4_t{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
        }
        if (left > 0 && left < 8) {   // the last columns, one by one
#pragma unroll 1
            for (int p = 0; p < PASSES; ++p) {
                if (!there(mb, p)) break;
                const uint32_t from = (read ^ (p * ROWS & 7) * 16) + p * ROWS * COLS * 4, row = mb * 16 + p * ROWS;
                const char* const r = res_at + (res_off + row * (uint32_t)a.ldr * (a.out32 ? 4u : 2u));
                char* const to = out_at + (out_off + row * (uint32_t)a.ldo * (a.out32 ? 4u : 2u));
#pragma unroll 1
                for (int i = 0; i < left; ++i) {
                    float x = *reinterpret_cast<const float*>(sums + ((from ^ (i >> 2) * 16u) + (i & 3) * 4));
                    if (a.residual) x += a.out32 ? reinterpret_cast<const float*>(r)[i] : bf16_lo(reinterpret_cast<const uint16_t*>(r)[i]);
                    if (a.out32) reinterpret_cast<float*>(to)[i] = x;
                    else reinterpret_cast<uint16_t*>(to)[i] = (uint16_t)pack_bf16x2(x, 0.f);
                }
            }
        }
        wavefront_lds_order();
    }
};

// v = acc[mb]; constants only, so that the accumulators stay in registers
template <int B, int MB, int NB>
__device__ __forceinline__ void row_of_blocks(int mb, const f32x4_t (&acc)[MB][NB], f32x4_t (&v)[NB])
{
    if (mb == B) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) v[nb] = acc[B][nb];
    } else if constexpr (B + 1 < MB) row_of_blocks<B + 1, MB, NB>(mb, acc, v);
}

// STAGED: operands that are not on 16 bytes come in through registers, a K step ahead, and are written to the next slot in front of its hand-over.
// RAGGED: the last K step is not whole.  ACT: there is an activation; a launch without one does not fetch the code of all of them (256 x 256
// tiles: 3 us of 19)
template <int BM, int BN, int SLOTS, int OCC, bool RAGGED, bool ACT, bool STAGED>
__global__ __launch_bounds__(256, OCC) void linear_tiled_kernel(LinearArgs a)
{
    using C = TileCfg<BM, BN, SLOTS>;
    constexpr int MB = C::MB, NB = C::NB, RPW = C::RPW, RX = C::RX;
    extern __shared__ uint4 lds4[];
    char* const lds = reinterpret_cast<char*>(lds4);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
    const int mt = (a.R + BM - 1) / BM, nt = (a.N + BN - 1) / BN, total = mt * nt, KT = (a.K + C::KS - 1) / C::KS;
    // workgroup b runs on XCD b mod 8: an XCD's tiles are consecutive ones, in bands of 8 row tiles, inside a band row tiles first
    const int per = gridDim.x >> 3, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
    const auto tile_at = [&](int it, int& m0, int& n0) -> bool {
        const int L = (it * 8 + xcd) * per + slot;
        if (L >= total) return false;
        constexpr int BAND = 8;
        const int band = L / (BAND * nt), h = min(BAND, mt - band * BAND), l = L - band * BAND * nt, ni = l / h;
        m0 = __builtin_amdgcn_readfirstlane((band * BAND + l - ni * h) * BM);
        n0 = __builtin_amdgcn_readfirstlane(ni * BN);
        return true;
    };

    // loads: where they come from, as byte offsets of this lane from the tile's rows
    const int ld_row = lane >> 3, ld_c = (lane & 7) ^ (lane >> 4);      // chunk of an even region's row; an odd one's is ld_c ^ 4
    const char *xi = nullptr, *wi = nullptr;
    uint32_t off[RPW];
    const auto aim = [&](int m0, int n0) __attribute__((always_inline)) {
        xi = reinterpret_cast<const char*>(a.x + (size_t)m0 * a.ldx);
        wi = reinterpret_cast<const char*>(static_cast<const uint16_t*>(a.w) + (size_t)n0 * a.ldw);
#pragma unroll
        for (int i = 0; i < RPW; ++i) {
            const int j = wave + C::NW * (i < RX ? i : i - RX), c = (j & 1) ? ld_c ^ 4 : ld_c;
            const int row = i < RX ? min(j * 8 + ld_row, a.R - 1 - m0) : min(j * 8 + ld_row, a.N - 1 - n0);
            off[i] = ((uint32_t)row * (uint32_t)(i < RX ? a.ldx : a.ldw) + c * 8) * 2u;
        }
    };
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    static_assert(!STAGED || SLOTS == 2, "one K step in registers");
    u32x4_t staged[STAGED ? RPW : 1];
    const auto issue = [&](int ks, int ring, int i) __attribute__((always_inline)) {
        const int j = wave + C::NW * (i < RX ? i : i - RX);
        if constexpr (STAGED) {
            const uint16_t* const p = reinterpret_cast<const uint16_t*>((i < RX ? xi : wi) + ks * (C::KS * 2) + off[i]);
            if (RAGGED && ks == KT - 1) staged[i] = load_part<8>(p, a.K - ks * C::KS - ((j & 1) ? ld_c ^ 4 : ld_c) * 8, a.K);
            else staged[i] = *reinterpret_cast<const u32x4_any2*>(p);
            return;
        }
        const char* const base = (i < RX ? xi : wi) + ks * (C::KS * 2);
        const uint32_t to = lds_base + (uint32_t)(ring * C::SLOT_BYTES + (i < RX ? 0 : BM * 128) + j * 1024);
        if (RAGGED && ks == KT - 1) {
            const char* src = base + off[i];
            if (ks * C::KS + ((j & 1) ? ld_c ^ 4 : ld_c) * 8 >= a.K) src = reinterpret_cast<const char*>(kZeros);
            load_to_lds(to, src);
        } else load_to_lds(to, base, off[i]);
    };
    const auto to_slot = [&](int ring) __attribute__((always_inline)) {
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < RPW; ++i)
                *reinterpret_cast<u32x4_t*>(lds + ring * C::SLOT_BYTES + (i < RX ? 0 : BM * 128) + (wave + C::NW * (i < RX ? i : i - RX)) * 1024 + lane * 16) = staged[i];
        }
    };
    const auto hand_over = [&]() __attribute__((always_inline)) {
        // this wavefront's loads into the next slot have landed (all but those into later ones), its reads have returned
        constexpr int LATER = (SLOTS - 2) * RPW;
        __builtin_amdgcn_s_waitcnt((LATER & 15) | ((LATER >> 4) << 14) | 0x0070);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // fragments: 16 rows x 32 k, 8 k per lane
    const int fr = lane & 15, kh = lane >> 4, sw = (fr >> 1) & 7;
    const uint32_t xa = (uint32_t)(wm * C::WTM + fr) * 128u, wa = (uint32_t)(BM + wn * C::WTN + fr) * 128u;
    const uint32_t ca = (uint32_t)(kh ^ sw) * 16u;                       // chunk of the first step of 32; the second's is ca ^ 64
    f32x4_t acc[MB][NB];
    bf16x8_t xf[2][MB], wf[2][NB];
    const auto frag = [&](int ring, int j, int f) __attribute__((always_inline)) {
        const char* base = lds + ring * C::SLOT_BYTES + (j ? ca ^ 64u : ca);
        // the first MFMA needs the first two
        const int x = f == 0 ? 0 : f <= NB ? -1 : f - NB, w = f == 0 ? -1 : f <= NB ? f - 1 : -1;
        if (x >= 0) xf[j][x < 0 ? 0 : x] = *reinterpret_cast<const bf16x8_t*>(base + xa + (x < 0 ? 0 : x) * 2048);
        else wf[j][w < 0 ? 0 : w] = *reinterpret_cast<const bf16x8_t*>(base + wa + (w < 0 ? 0 : w) * 2048);
    };

    int m0, n0, it = 0;
    if (!tile_at(0, m0, n0)) return;
    aim(m0, n0);
    int ring = 0, ki = 0, next_m0 = m0, next_n0 = n0;   // ki: the K step whose loads start at the next hand-over
    bool more = true;                                    // there is a tile behind the one that is multiplied
    const auto advance = [&]() __attribute__((always_inline)) {
        if (ki == KT) {
            more = tile_at(it + 1, next_m0, next_n0);
            if (more) aim(next_m0, next_n0);     // the last tile's loads go round to its own first K steps, and are not used
            ki = 0;
        }
    };
#pragma unroll
    for (int st = 0; st < SLOTS - 1; ++st) {
#pragma unroll
        for (int i = 0; i < RPW; ++i) issue(ki, st, i);
        ++ki;
    }
    to_slot(0);
    hand_over();
    // the last slot's loads start as every later one's do
    advance();
#pragma unroll
    for (int p = 0; p < C::TAIL; ++p)
        if (C::load_at(p) >= 0) issue(ki, SLOTS - 1, C::load_at(p) < 0 ? 0 : C::load_at(p));
#pragma unroll
    for (int f = 0; f < MB + NB; ++f) frag(0, 0, f);
    for (;;) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        // the compiler does not know the hand-written MFMAs' latencies: wait states around them
        SB();
        asm volatile("s_nop 7");
        SB();
        for (int kt = 0; kt < KT; ++kt) {
            const int other = ring == SLOTS - 1 ? 0 : ring + 1, last = ring == 0 ? SLOTS - 1 : ring - 1;
#pragma unroll
            for (int p = 0; p < C::M; ++p) {
                const int j = p / (MB * NB), q = p % (MB * NB), nb = q / MB, mb = (nb & 1) ? MB - 1 - q % MB : q % MB;
                if (p == C::HO) {
                    ++ki;
                    advance();
                    to_slot(other);
                    hand_over();
                }
                asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[mb][nb]) : "v"(wf[j][nb]), "v"(xf[j][mb]));
                if (j == 0) {
                    if (q % C::RD == 0 && q / C::RD < MB + NB) frag(ring, 1, q / C::RD);
                } else if (p >= C::HO) {
                    constexpr int RS = C::TAIL / (MB + NB);
                    if ((p - C::HO) % RS == 0 && (p - C::HO) / RS < MB + NB) frag(other, 0, (p - C::HO) / RS);
                }
                if (p >= C::HO) {
                    if (C::load_at(p - C::HO) >= 0) issue(ki, ring, C::load_at(p - C::HO) < 0 ? 0 : C::load_at(p - C::HO));
                } else if (C::load_at(p + C::TAIL) >= 0) issue(ki, last, C::load_at(p + C::TAIL) < 0 ? 0 : C::load_at(p + C::TAIL));
                SB();
            }
            ring = other;
        }
        SB();
        asm volatile("s_nop 15");
        asm volatile("s_nop 15");
        SB();
        // a row of blocks at a time, in a loop with one body: a body per row is 80 KB of code, more than the instruction cache holds
        const TileEpilogue<MB, C::WTN, ACT> e(a, lds + SLOTS * C::SLOT_BYTES + wave * C::SUM_BYTES, lane, m0 + wm * C::WTM, n0 + wn * C::WTN);
        typename TileEpilogue<MB, C::WTN, ACT>::Residual ahead;
        if (a.residual) e.fetch(0, ahead);
#pragma unroll 1
        for (int mb = 0; mb < MB; ++mb) {
            const typename TileEpilogue<MB, C::WTN, ACT>::Residual res = ahead;
            if (a.residual && mb + 1 < MB) e.fetch(mb + 1, ahead);
            f32x4_t v[NB];
            row_of_blocks<0, MB, NB>(mb, acc, v);
            e.store(mb, v, res);
        }
        if (!more) break;
        m0 = next_m0;
        n0 = next_n0;
        ++it;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);   // no load may land in LDS that is another workgroup's by then
}

template <int BM, int BN, int SLOTS, int OCC, bool RAGGED, bool ACT, bool STAGED>
hipError_t launch_tiled_as(const LinearArgs& a, int n_cu, hipStream_t s)
{
    using C = TileCfg<BM, BN, SLOTS>;
    static_assert(C::LDS_BYTES * OCC <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> told{0};
    const hipError_t e = allow_lds(&linear_tiled_kernel<BM, BN, SLOTS, OCC, RAGGED, ACT, STAGED>, C::LDS_BYTES, told);
    if (e != hipSuccess) return e;
    const long long total = (long long)((a.R + BM - 1) / BM) * ((a.N + BN - 1) / BN);
    if (total > 0x3fffffffll) return hipErrorInvalidValue;
    // as few workgroups as it takes for as many rounds, the same number on every XCD
    const long long wgs = (long long)n_cu * OCC, rounds = (total + wgs - 1) / wgs;
    const int grid = (int)(((total + rounds - 1) / rounds + 7) / 8 * 8);
    hipLaunchKernelGGL((linear_tiled_kernel<BM, BN, SLOTS, OCC, RAGGED, ACT, STAGED>), dim3(grid), dim3(256), C::LDS_BYTES, s, a);
    return hipGetLastError();
}

template <int BM, int BN, int SLOTS, int OCC, bool STAGED = false>
hipError_t launch_tiled(const LinearArgs& a, int n_cu, hipStream_t s)
{
    // (staged: K is seldom whole)
    if constexpr (!STAGED) {
        if (a.act == kActNone && a.K % 64 == 0) return launch_tiled_as<BM, BN, SLOTS, OCC, false, false, false>(a, n_cu, s);
        if (a.K % 64 == 0) return launch_tiled_as<BM, BN, SLOTS, OCC, false, true, false>(a, n_cu, s);
    }
    return a.act == kActNone ? launch_tiled_as<BM, BN, SLOTS, OCC, true, false, STAGED>(a, n_cu, s) : launch_tiled_as<BM, BN, SLOTS, OCC, true, true, STAGED>(a, n_cu, s);
}

// What a tile costs, us: `fixed` and, per K step, `alone` where most compute units have none, `full` where all have (power and
// L2 are shared).  Fitted to launches of 256 x 256 to 16384 x 5120 results, K from 256 to 8192.
struct Tiling { int rows, cols, slots, per_cu; double alone, full, fixed; };
constexpr Tiling kTilings[] = {
    {256, 256, 2, 1, 1.02, 1.40, 12.0}, {256, 192, 2, 1, 0.84, 1.13, 9.5}, {192, 256, 2, 1, 0.85, 1.13, 9.0},
    {128, 128, 4, 1, 0.33, 0.44, 5.0}, {64, 64, 4, 2, 0.15, 0.37, 1.2}};

// a launch lasts as many rounds as its busiest compute unit has tiles
double tiled_us(const Tiling& t, const LinearArgs& a, int n_cu)
{
    const double tiles = (double)((a.R + t.rows - 1) / t.rows) * ((a.N + t.cols - 1) / t.cols), slots = (double)n_cu * t.per_cu;
    const double rounds = std::ceil(tiles / slots), fill = tiles / (rounds * slots);
    return rounds * ((a.K + 63) / 64 * (t.alone + (t.full - t.alone) * fill) + t.fixed);
}

// the tiling of kTilings that costs least
int cheapest_tiling(const LinearArgs& a, int n_cu)
{
    int best = 0;
    double us = 0.0;
    for (int i = 0; i < (int)(sizeof kTilings / sizeof *kTilings); ++i) {
        const double t = tiled_us(kTilings[i], a, n_cu);
        if (kTilings[i].slots <= (a.K + 63) / 64 && (us == 0.0 || t < us)) { us = t; best = i; }
    }
    return best;
}

// The largest of the split tiles that still gives enough compute units work: half of them, three quarters where every tile also takes fp32
// weights apart.  64 x 32 / 64 x 16 / 32 x 16 / 16 x 16 tiles, us: 64 x 5120 x 1536 10 / 12 / 15 / 13; 33, 64 x 2048 x 1408 7.2 / 6.2 / 5.2 / 5.4,
// 7.3 / 6.4 / 5.2 / 5.5; 64 x 1536 x 5120 22 / 18 / 13 / 14; 24 x 1536 x 5120 18 / 15 / 12 / 9; 17, 32 x 5120 x 1536 8.9 / 11 / 10 / 8.9, 9.2 / 11 / 11 / 9.7;
// fp32 weights, 4096 x 128 x 4096 27 / 32 / 43 / 62, 1024 x 256 x 4096 23 / 16 / 23 / 33, 256 x 160 x 5120 25 / 17 / 12 / 10.  (Of 33 to 64 rows the
// rule takes 64 x 16 where 32 x 16 is up to a fifth faster: half of the compute units is too few there.)  64 x 32 with four wavefronts instead of
// eight, many tiles: 4096 x 256 x 2048 25 / 28, 8192 x 256 x 4096 87 / 94; 4096 x 128 x 4096, few, 31 / 27.
int split_kernel(const LinearArgs& a, int n_cu)
{
    const auto tiles = [&](int mb, int nb) { return (double)((a.R + mb * 16 - 1) / (mb * 16)) * ((a.N + nb * 16 - 1) / (nb * 16)); };
    const double enough = a.w32 ? 0.75 * n_cu : 0.5 * n_cu;
    if (a.R > 32 && tiles(4, 2) >= 2 * n_cu) return kLinearSplit64x32by4;
    if (a.R > 32 && tiles(4, 2) >= enough) return kLinearSplit64x32;
    if (a.R > 32 && tiles(4, 1) >= enough) return kLinearSplit64x16;
    if (a.R > 16 && tiles(2, 1) >= enough) return kLinearSplit32x16;
    return kLinearSplit16x16;
}

}  // namespace

int linear_kernel(const LinearArgs& a, int n_cu)
{
    const auto tiles = [&](int edge) { return (double)((a.R + edge - 1) / edge) * ((a.N + edge - 1) / edge); };
    // Few blocks of 16 x 16 for a matrix instruction, and little to multiply.  Rows / split, us: 1, 16, 33 x 160 x 5120, fp32 weights, 3.1 / 8.6,
    // 5.1 / 8.6, 6.5 / 8.7; 64, 256 x 128 x 4096 6.6 / 7.5, 17 / 9.1; bf16 weights, 1, 8 x 2048 x 1408 3.6 / 3.8, 7.6 / 3.9.
    const double products = (double)a.R * a.N * a.K;
    if ((products <= 40e6 && tiles(16) < n_cu / 2) || products <= 3e6) return a.R <= 8 ? kLinearRows1x1 : a.R <= 16 ? kLinearRows4x1 : kLinearRows4x2;
    // The tiled kernels move 16 bytes at a time, and are a K step ahead at least.  Of few tiles, each a compute unit's, a long K is better shared:
    // tiled / split, us: 64 x 1536 x 5120 17 / 9.7; 64 x 5120 x 2048 9.8 / 9.5, 256 x 2048 x 2048 9.6 / 12.
    const bool by_16 = !a.w32 && a.K > 64 && a.K % 8 == 0 && a.ldx % 8 == 0 && a.ldw % 8 == 0 && !((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15);
    if (by_16 && a.R > 64 && tiles(64) >= n_cu / 4) return kLinearTiled + cheapest_tiling(a, n_cu);
    // Operands that are not on 16 bytes: 64 x 64 tiles / 128 x 64 tiles / split, us: 1531 x 1409 x 2049 39 / 43 / 49, 3112 x 839 x 182 8.9 / 11 / 12,
    // 8192 x 2048 x 2049 197 / 149 / 260, 16384 x 5120 x 1001 486 / 426 / 755; of few tiles 300 x 1409 x 2049 27 / 37 / 14.
    if (!a.w32 && !by_16 && a.K > 64) {
        if (2 * tiles(128) >= 4 * n_cu) return kLinearStaged128x64;
        if (tiles(64) >= 1.5 * n_cu) return kLinearStaged64x64;
    }
    return split_kernel(a, n_cu);
}

hipError_t launch_linear(const LinearArgs& a, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.N < 1 || a.K < 1) return hipErrorInvalidValue;
    switch (linear_kernel(a, n_cu)) {
    case kLinearRows1x1: return launch_rows<1, 1>(a, s);
    case kLinearRows4x1: return launch_rows<4, 1>(a, s);
    case kLinearRows4x2: return launch_rows<4, 2>(a, s);
    case kLinearTiled + 0: return launch_tiled<256, 256, 2, 1>(a, n_cu, s);
    case kLinearTiled + 1: return launch_tiled<256, 192, 2, 1>(a, n_cu, s);
    case kLinearTiled + 2: return launch_tiled<192, 256, 2, 1>(a, n_cu, s);
    case kLinearTiled + 3: return launch_tiled<128, 128, 4, 1>(a, n_cu, s);
    case kLinearTiled + 4: return launch_tiled<64, 64, 4, 2>(a, n_cu, s);
    case kLinearStaged128x64: return launch_tiled<128, 64, 2, 2, true>(a, n_cu, s);
    case kLinearStaged64x64: return launch_tiled<64, 64, 2, 3, true>(a, n_cu, s);
    case kLinearSplit64x32by4: return launch_split<4, 2, 4>(a, s);
    case kLinearSplit64x32: return launch_split<4, 2, 8>(a, s);
    case kLinearSplit64x16: return launch_split<4, 1, 8>(a, s);
    case kLinearSplit32x16: return launch_split<2, 1, 16>(a, s);
    default: return launch_split<1, 1, 16>(a, s);
    }
}

}  // namespace moe_ep
