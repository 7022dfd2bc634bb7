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

#define SB() __builtin_amdgcn_sched_barrier(0)

__device__ const uint4 kZeros[4] = {};   // what a lane fetches that is beyond its row's end

// Many rows and columns: tiles of BM rows x BN columns through LDS, 2 x 2 wavefronts.  A K step is 64 elements, rows of 128 bytes
// whose 16-byte chunks are XOR-swizzled by the row, so that fragment reads meet no bank twice; global_load_lds brings them in, a ring of
// two slots.  A workgroup takes tiles in turn; the loads run a K step ahead of the multiplications, across tiles too.
template <int BM, int BN>
struct TileCfg {
    static constexpr int KS = 64, NW = 4, SLOTS = 2;
    static constexpr int WTM = BM / 2, WTN = BN / 2, MB = WTM / 16, NB = WTN / 16;
    static constexpr int RX = BM / 8 / NW, RW = BN / 8 / NW, RPW = RX + RW;   // 1 KB regions (8 rows) a wavefront loads per K step
    static constexpr int SLOT_BYTES = (BM + BN) * KS * 2;
    static constexpr int LANES = WTN / 8, SUM_BYTES = 16 * WTN * 4;           // epilogue: 8 columns a lane; a wavefront's row of blocks in fp32
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

// The results of 16 rows x 8 * LANES columns that a wavefront holds in LDS as fp32 (16-byte chunks XOR-swizzled by the row): bias, activation,
// residual, rounding, stores of whole pieces of a row.  A lane has 8 consecutive columns n.. of every (64 / LANES)th row from m on.
template <int LANES>
__device__ __forceinline__ void finish_rows(const LinearArgs& a, const char* sums, int lane, int m, int n, const float bias[8])
{
    constexpr int ROWS = 64 / LANES;
    const int c = lane % LANES, left = a.N - n;
#pragma unroll 1
    for (int r = lane / LANES; r < 16; r += ROWS) {
        if (m + r >= a.R || left <= 0) continue;
        const char* row = sums + r * LANES * 32;
        const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(row + ((2 * c) ^ (r & 7)) * 16);
        const f32x4_t hi = *reinterpret_cast<const f32x4_t*>(row + ((2 * c + 1) ^ (r & 7)) * 16);
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += bias[i];
        if (a.act != kActNone) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = activate(a.act, v[i]);
        }
        if (a.residual) {
            const size_t from = (size_t)(m + r) * a.ldr + n;
            if (a.out32) {
                const float* p = static_cast<const float*>(a.residual) + from;
                if (left >= 8) {
                    const f32x4_t x = *reinterpret_cast<const f32x4_any4*>(p), y = *reinterpret_cast<const f32x4_any4*>(p + 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) { v[i] += x[i]; v[i + 4] += y[i]; }
                } else for (int i = 0; i < 8; ++i) if (i < left) v[i] += p[i];
            } else {
                const bf16x8_t x = load8(static_cast<const uint16_t*>(a.residual) + from, left);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += (float)x[i];
            }
        }
        const size_t at = (size_t)(m + r) * a.ldo + n;
        if (a.out32) {
            float* p = static_cast<float*>(a.out) + at;
            if (left >= 8) {
                *reinterpret_cast<f32x4_any4*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4_any4*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
            } else for (int i = 0; i < 8; ++i) if (i < left) p[i] = v[i];
        } else {
            uint16_t* p = static_cast<uint16_t*>(a.out) + at;
            const u32x4_t o = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
            if (left >= 8) *reinterpret_cast<u32x4_any2*>(p) = o;
            else for (int i = 0; i < 8; ++i) if (i < left) p[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// RAGGED: the last K step is not whole
template <int BM, int BN, int OCC, bool RAGGED>
__global__ __launch_bounds__(256, OCC) void linear_tiled_kernel(LinearArgs a)
{
    using C = TileCfg<BM, BN>;
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
    const auto issue = [&](int ks, int ring, int i) __attribute__((always_inline)) {
        const int j = wave + C::NW * (i < RX ? i : i - RX);
        const char* src = (i < RX ? xi : wi) + ks * (C::KS * 2) + off[i];
        if (RAGGED && ks == KT - 1 && ks * C::KS + ((j & 1) ? ld_c ^ 4 : ld_c) * 8 >= a.K) src = reinterpret_cast<const char*>(kZeros);
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(src), reinterpret_cast<uint4*>(lds + ring * C::SLOT_BYTES + (i < RX ? 0 : BM * 128) + j * 1024), 16, 0, 0);
    };
    const auto hand_over = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0): this wavefront's loads have landed, its reads have returned
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
    int ring = 0, ki = 1, next_m0 = m0, next_n0 = n0;   // ki: the K step whose loads start at the next hand-over
    bool more = true;                                    // there is a tile behind the one that is multiplied
#pragma unroll
    for (int i = 0; i < RPW; ++i) issue(0, 0, i);
    hand_over();
    // K step 1 (or the next tile's first one) starts as every later one does
    const auto advance = [&]() __attribute__((always_inline)) {
        if (ki == KT) {
            more = tile_at(it + 1, next_m0, next_n0);
            if (more) aim(next_m0, next_n0);     // the last tile's loads go round to its own first K step, and are not used
            ki = 0;
        }
    };
    advance();
#pragma unroll
    for (int p = 0; p < C::TAIL; ++p)
        if (C::load_at(p) >= 0) issue(ki, 1, C::load_at(p) < 0 ? 0 : C::load_at(p));
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
            const int other = ring ^ 1;
#pragma unroll
            for (int p = 0; p < C::M; ++p) {
                const int j = p / (MB * NB), q = p % (MB * NB), nb = q / MB, mb = (nb & 1) ? MB - 1 - q % MB : q % MB;
                if (p == C::HO) {
                    ++ki;
                    advance();
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
                } else if (C::load_at(p + C::TAIL) >= 0) issue(ki, other, C::load_at(p + C::TAIL) < 0 ? 0 : C::load_at(p + C::TAIL));
                SB();
            }
            ring = other;
        }
        SB();
        asm volatile("s_nop 15");
        asm volatile("s_nop 15");
        SB();
// A lane holds row (lane & 15) of each block and 4 consecutive columns of it.  A row of blocks at a time goes through LDS, so that a
        // store carries whole pieces of a row and the code of the epilogue is there once.
        char* const sums = lds + C::SLOTS * C::SLOT_BYTES + wave * C::SUM_BYTES;
        const int n = n0 + wn * C::WTN + (lane % C::LANES) * 8;
        float bias[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = a.bias && n + i < a.N ? a.bias[n + i] : 0.f;
#pragma unroll 1
        for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
            for (int b = 0; b < MB; ++b)
                if (b == mb) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        *reinterpret_cast<f32x4_t*>(sums + fr * (NB * 64) + ((nb * 4 + kh) ^ (fr & 7)) * 16) = acc[b][nb];
                }
            wavefront_lds_order();
            finish_rows<C::LANES>(a, sums, lane, m0 + wm * C::WTM + mb * 16, n, bias);
            wavefront_lds_order();
        }
        if (!more) break;
        m0 = next_m0;
        n0 = next_n0;
        ++it;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);   // no load may land in LDS that is another workgroup's by then
}

template <int BM, int BN, int OCC, bool RAGGED>
hipError_t launch_tiled_k(const LinearArgs& a, int n_cu, hipStream_t s)
{
    using C = TileCfg<BM, BN>;
    static_assert(C::LDS_BYTES * OCC <= 160 * 1024, "LDS of a compute unit");
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&linear_tiled_kernel<BM, BN, OCC, RAGGED>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES);
    if (e != hipSuccess) return e;
    const long long total = (long long)((a.R + BM - 1) / BM) * ((a.N + BN - 1) / BN);
    if (total > 0x3fffffffll) return hipErrorInvalidValue;
    // as few workgroups as it takes for as many rounds, the same number on every XCD
    const long long wgs = (long long)n_cu * OCC, rounds = (total + wgs - 1) / wgs;
    const int grid = (int)(((total + rounds - 1) / rounds + 7) / 8 * 8);
    hipLaunchKernelGGL((linear_tiled_kernel<BM, BN, OCC, RAGGED>), dim3(grid), dim3(256), C::LDS_BYTES, s, a);
    return hipGetLastError();
}

template <int BM, int BN, int OCC>
hipError_t launch_tiled(const LinearArgs& a, int n_cu, hipStream_t s)
{
    return a.K % TileCfg<BM, BN>::KS ? launch_tiled_k<BM, BN, OCC, true>(a, n_cu, s) : launch_tiled_k<BM, BN, OCC, false>(a, n_cu, s);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.N < 1 || a.K < 1) return hipErrorInvalidValue;
    // the tiled kernel moves 16 bytes at a time
    // (and is always one K step ahead: two at least)
    const bool by_16 = !a.w32 && a.K > 64 && a.K % 8 == 0 && a.ldx % 8 == 0 && a.ldw % 8 == 0 && !((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15);
    if (by_16 && a.R > 64) {
        const long long big = (long long)((a.R + 255) / 256) * ((a.N + 255) / 256);
        if (big >= n_cu) return launch_tiled<256, 256, 1>(a, n_cu, s);
        return launch_tiled<128, 128, 2>(a, n_cu, s);
    }
    if (a.R <= 16) return launch_split<1, 1, 16>(a, s);
    if (a.R <= 32) return launch_split<2, 1, 16>(a, s);
    return launch_split<4, 2, 8>(a, s);
}

}  // namespace moe_ep
