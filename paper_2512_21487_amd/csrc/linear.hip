// Matrix product with an epilogue: out = act(x W^T + bias) + residual, for the gate's scores (weights in fp32) and for dense layers.
// Both operands are K-contiguous, which is what the bf16 matrix instructions want per lane; the weight rows are the first operand, so
// that a lane ends up with four consecutive output columns of one row.  Sums, bias, activation and residual are fp32; a result is
// rounded once.
//
// fp32 weights are three bf16 numbers each, 8 mantissa bits at a time cut off the top (24 together: all of them), and a product is three
// matrix instructions: as exact as fp32 multiplications at 5 times their rate.
#include "common.h"

namespace moe_ep {

namespace {

// 16 bytes from an address that only the type of the elements aligns
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float gelu_tanh_f(float z)
{
    // 0.5 z (1 + tanh(u)) = z / (1 + exp(-2u)),  u = sqrt(2 / pi) (z + 0.044715 z^3)
    const float u = 0.7978845608028654f * (z + 0.044715f * z * z * z);
    return z / (1.0f + expf(-2.0f * u));
}

__device__ __forceinline__ float activate(int act, float z)
{
    switch (act) {
    case kActRelu: return z < 0.f ? 0.f : z;   // a NaN stays one
    case kActSilu: return z / (1.0f + expf(-z));
    case kActGelu: return 0.5f * z * (1.0f + erff(z * 0.7071067811865476f));
    case kActGeluTanh: return gelu_tanh_f(z);
    default: return z;
    }
}

// four consecutive columns of a row: bias, activation, residual, rounding, store
__device__ __forceinline__ void finish(const LinearArgs& a, int m, int n, f32x4_t v)
{
    const int left = a.N - n;
    if (m >= a.R || left <= 0) return;
    const bool whole = left >= 4;
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += a.bias[n + (whole ? i : min(i, left - 1))];
    }
    if (a.act != kActNone) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = activate(a.act, v[i]);
    }
    const size_t at = (size_t)m * a.ldo + n;
    if (a.residual) {
        const size_t from = (size_t)m * a.ldr + n;
        if (a.out32) {
            const float* r = static_cast<const float*>(a.residual) + from;
            if (whole) v += *reinterpret_cast<const f32x4_any4*>(r);
            else for (int i = 0; i < left; ++i) v[i] += r[i];
        } else {
            const uint16_t* r = static_cast<const uint16_t*>(a.residual) + from;
            for (int i = 0; i < 4; ++i) if (i < left) v[i] += __uint_as_float((uint32_t)r[i] << 16);
        }
    }
    if (a.out32) {
        float* o = static_cast<float*>(a.out) + at;
        if (whole) *reinterpret_cast<f32x4_any4*>(o) = v;
        else for (int i = 0; i < left; ++i) o[i] = v[i];
    } else {
        uint16_t* o = static_cast<uint16_t*>(a.out) + at;
        const uint32_t p[2] = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        for (int i = 0; i < 4; ++i) if (i < left) o[i] = (uint16_t)(p[i >> 1] >> (16 * (i & 1)));
    }
}

// 8 elements of a row from element k on, zeros from the row's end on; p: element k
__device__ __forceinline__ bf16x8_t load8(const uint16_t* p, int left)
{
    if (left >= 8) return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_any2*>(p));
    uint32_t v[4] = {0, 0, 0, 0};
    for (int i = 0; i < 8; ++i) if (i < left) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    const u32x4_t u = {v[0], v[1], v[2], v[3]};
    return __builtin_bit_cast(bf16x8_t, u);
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

// Few rows or few columns: both operands go from memory straight into the lanes that multiply them, and the wavefronts of a workgroup
// take K steps of 64 in turn; their sums are added up in LDS, in the order of the wavefronts.  MB x NB blocks of 16 rows x 16 columns.
template <int MB, int NB, int WAVES, bool W32>
__global__ __launch_bounds__(WAVES * 64) void linear_split_kernel(LinearArgs a)
{
    constexpr int KS = 64;
    __shared__ f32x4_t s_sum[WAVES][MB * NB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // tiles of one XCD (workgroup number mod 8) are consecutive ones
    const int mt = (a.R + MB * 16 - 1) / (MB * 16), nt = (a.N + NB * 16 - 1) / (NB * 16);
    const long long total = (long long)mt * nt, per = (total + 7) / 8, L = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || L >= total) return;
    const int m0 = (int)(a.rows_first ? L % mt : L / nt) * (MB * 16), n0 = (int)(a.rows_first ? L / mt : L % nt) * (NB * 16);
    const int row = lane & 15, kq = (lane >> 4) * 8;

    const uint16_t* xp[MB];
    const char* wp[NB];
    constexpr int WB = W32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < MB; ++i) xp[i] = a.x + (size_t)min(m0 + i * 16 + row, a.R - 1) * a.ldx + kq;
#pragma unroll
    for (int i = 0; i < NB; ++i) wp[i] = static_cast<const char*>(a.w) + ((size_t)min(n0 + i * 16 + row, a.N - 1) * a.ldw + kq) * WB;

    f32x4_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int k0 = wave * KS; k0 < a.K; k0 += WAVES * KS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + h * 32, left = a.K - k - kq;
            bf16x8_t xf[MB];
#pragma unroll
            for (int i = 0; i < MB; ++i) xf[i] = load8(xp[i] + k, left);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if constexpr (W32) {
                    bf16x8_t part[3];
                    split3(load8(reinterpret_cast<const float*>(wp[j]) + k, left), part);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
#pragma unroll
                        for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[p], xf[i], acc[i][j], 0, 0, 0);
                } else {
                    const bf16x8_t wf = load8(reinterpret_cast<const uint16_t*>(wp[j]) + k, left);
#pragma unroll
                    for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[i], acc[i][j], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) s_sum[wave][i * NB + j][lane] = acc[i][j];
    __syncthreads();
    // neighbouring threads: neighbouring columns
    for (int q = threadIdx.x; q < MB * NB * 64; q += WAVES * 64) {
        const int r = q / (NB * 4), c = q % (NB * 4), b = (r / 16) * NB + c / 4, l = (c & 3) * 16 + (r & 15);
        f32x4_t v = s_sum[0][b][l];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_sum[w][b][l];
        finish(a, m0 + r, n0 + c * 4, v);
    }
}

template <int MB, int NB, int WAVES>
hipError_t launch_split(LinearArgs a, hipStream_t s)
{
    const long long mt = (a.R + MB * 16 - 1) / (MB * 16), nt = (a.N + NB * 16 - 1) / (NB * 16), per = (mt * nt + 7) / 8;
    if (per * 8 > 0x7fffffffll) return hipErrorInvalidValue;
    // an XCD's tiles share the rows of the larger operand through its L2
    a.rows_first = (double)a.N * a.K * (a.w32 ? 4 : 2) > (double)a.R * a.K * 2;
    if (a.w32) hipLaunchKernelGGL((linear_split_kernel<MB, NB, WAVES, true>), dim3((unsigned)(per * 8)), dim3(WAVES * 64), 0, s, a);
    else hipLaunchKernelGGL((linear_split_kernel<MB, NB, WAVES, false>), dim3((unsigned)(per * 8)), dim3(WAVES * 64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, int n_cu, hipStream_t s)
{
    (void)n_cu;
    if (a.R <= 0) return hipSuccess;
    if (a.N < 1 || a.K < 1) return hipErrorInvalidValue;
    if (a.R <= 16) return launch_split<1, 1, 16>(a, s);
    if (a.R <= 32) return launch_split<2, 1, 16>(a, s);
    return launch_split<4, 2, 8>(a, s);
}

}  // namespace moe_ep
