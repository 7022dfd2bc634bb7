// Low-rank adapters of many requests beside a shared projection: act(x W^T + bias + scale_a (x A_a^T) B_a^T) + residual, a = index[row].
// Two launches.  The first makes scale_a x A_a^T of every row with an adapter, and for every row tile of the second the list of its rows' adapters.  The
// second is the product's own kernel (linear_kernels.h), whose reduction goes on behind K with these products and B_a: the
// wide result is neither written twice nor read again.
#include "linear_kernels.h"

namespace moe_ep {

namespace {

// The adapters of up to 64 rows, one a lane, in the order of their first rows: next() gives one after the other, and which lanes have it.
struct Distinct {
    int mine;
    unsigned long long left;
    __device__ __forceinline__ explicit Distinct(int adapter) : mine(adapter), left(__ballot(adapter >= 0)) {}
    __device__ __forceinline__ bool next(int& adapter, unsigned long long& who)
    {
        if (!left) return false;
        adapter = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
        who = __ballot(mine == adapter);
        left &= ~who;
        return true;
    }
};

// the list of a tile of up to 256 rows, by one wavefront
__device__ __forceinline__ void make_list(const LinearArgs& a, const AdapterArgs& x, long long tile, int lane)
{
    int32_t* const list = x.lists + tile * adapter_list(x.tile);
    const int masks = (x.tile + 31) / 32;
    int mine[4], count = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long row = tile * x.tile + i * 64 + lane;
        mine[i] = i * 64 + lane < x.tile && row < a.R ? adapter_of(x, (int)row) : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        Distinct d(mine[i]);
        int adapter;
        unsigned long long who[4] = {0, 0, 0, 0};
        while (d.next(adapter, who[i])) {
#pragma unroll
            for (int j = i + 1; j < 4; ++j) {
                who[j] = __ballot(mine[j] == adapter);
                if (mine[j] == adapter) mine[j] = -1;
            }
            // lane 0 writes the number, lane 1 + m the rows 32 m ..
            uint32_t v = (uint32_t)adapter;
#pragma unroll
            for (int m = 0; m < 8; ++m)
                if (lane == 1 + m) v = (uint32_t)(who[m >> 1] >> (m & 1) * 32);
            if (lane <= masks) list[1 + count * (1 + masks) + lane] = (int32_t)v;
            ++count;
        }
    }
    if (lane == 0) list[0] = count;
}

// A wavefront's 16 rows x 16 ranks of sums: a lane has 4 consecutive ranks of its row, r the first.  They are written as `parts` bf16 numbers each, 8 bits cut off the top at a
// time and the last rounded: two leave 2^-17 of the sum, which is 2^-8 of what rounding the result to bf16 leaves, three 2^-25 (results in fp32).
__device__ __forceinline__ void store_low(const AdapterArgs& x, long long row, int r, f32x4_t v)
{
    uint16_t* const to = x.low + row * adapter_pitch(x.width) + r;
    for (int p = 0; p < x.parts; ++p) {
        u32x2_t u;
        if (p + 1 == x.parts) u = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else {
            u = u32x2_t{upper_halves(v[0], v[1]), upper_halves(v[2], v[3])};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] -= __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
        }
        *reinterpret_cast<u32x2_t*>(to + p * x.rank) = u;
    }
}

// x A_a^T of MB * 16 rows and NB * 16 ranks: the wavefronts take K steps of 64 in turn, as in linear_split_kernel.  A tile's adapters are dealt out to `groups` workgroups.
template <int MB, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void adapters_down_kernel(LinearArgs a, AdapterArgs x, int list_tiles, int groups)
{
    using C = SplitCfg<MB, NB, false>;
    constexpr int KS = C::KS;
    extern __shared__ uint4 lds4[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long list_groups = (list_tiles + WAVES - 1) / WAVES, b = workgroup() - list_groups;
    if (b < 0) {
        const long long tile = workgroup() * WAVES + wave;
        if (tile < list_tiles) make_list(a, x, tile, lane);
        return;
    }
    const int blocks = (x.rank + NB * 16 - 1) / (NB * 16);
    const int r0 = (int)(b % blocks) * (NB * 16), group = (int)(b / blocks % groups);
    const long long m0 = b / blocks / groups * (MB * 16);
    if (m0 >= a.R) return;
    char* const own = reinterpret_cast<char*>(lds4) + wave * C::BYTES;
    const int xr = lane >> 3, xc = lane & 7, row = lane & 15, kh = lane >> 4, sw = (row >> 1) & 7;
    // the zeros behind every row, one with an adapter or not
    if (b % blocks == 0 && group == 0 && wave == 0 && lane < MB * 16 && m0 + lane < a.R)
        *reinterpret_cast<u32x4_t*>(x.low + (m0 + lane) * adapter_pitch(x.width) + x.width) = u32x4_t{0, 0, 0, 0};
    Distinct tile(lane < MB * 16 && m0 + lane < a.R ? adapter_of(x, (int)(m0 + lane)) : -1);
    int adapter;
    unsigned long long who;
    for (int at = 0; tile.next(adapter, who); ++at) {
        if (at % groups != group) continue;
        const uint16_t* const w0 = x.down + ((size_t)adapter * x.rank + r0) * a.K;
        const uint16_t* const x0 = a.x + (size_t)m0 * a.ldx;
        struct Step { u32x4_t x[C::XL], w[C::WL]; } f;
        const auto load = [&](int step) __attribute__((always_inline)) {
            const int left = a.K - step * KS;
#pragma unroll
            for (int i = 0; i < C::WL; ++i) {
                f.w[i] = u32x4_t{0, 0, 0, 0};
                if (r0 + i * 8 + xr < x.rank) f.w[i] = load_part<8>(w0 + (size_t)(i * 8 + xr) * a.K + step * KS + xc * 8, left - xc * 8, a.K);
            }
#pragma unroll
            for (int i = 0; i < C::XL; ++i) {
                f.x[i] = u32x4_t{0, 0, 0, 0};
                if (who >> (i * 8 + xr) & 1) f.x[i] = load_part<8>(x0 + (size_t)(i * 8 + xr) * a.ldx + step * KS + xc * 8, left - xc * 8, a.K);
            }
        };
        f32x4_t acc[MB][NB];
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const int steps = (a.K + KS - 1) / KS;
        if (wave < steps) load(wave);
        for (int st = wave; st < steps; st += WAVES) {
#pragma unroll
            for (int i = 0; i < C::WL; ++i) *reinterpret_cast<u32x4_t*>(own + C::X_BYTES + xr * 128 + i * 1024 + (xc ^ (((i * 8 + xr) >> 1) & 7)) * 16) = f.w[i];
#pragma unroll
            for (int i = 0; i < C::XL; ++i) *reinterpret_cast<u32x4_t*>(own + xr * 128 + i * 1024 + (xc ^ (((i * 8 + xr) >> 1) & 7)) * 16) = f.x[i];
            wavefront_lds_order();
            if (st + WAVES < steps) load(st + WAVES);
            SB();   // or the compiler moves loads behind the products
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8_t xs[MB];
#pragma unroll
                for (int i = 0; i < MB; ++i) xs[i] = *reinterpret_cast<const bf16x8_t*>(own + (i * 16 + row) * 128 + ((h * 4 + kh) ^ sw) * 16);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const bf16x8_t w = *reinterpret_cast<const bf16x8_t*>(own + C::X_BYTES + (j * 16 + row) * 128 + ((h * 4 + kh) ^ sw) * 16);
#pragma unroll
                    for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, xs[i], acc[i][j], 0, 0, 0);
                }
            }
            wavefront_lds_order();
        }
        // a wavefront's operands make room for its sums
        f32x4_t* const sums = reinterpret_cast<f32x4_t*>(own) + lane;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) sums[(i * NB + j) * 64] = acc[i][j];
        __syncthreads();
        const float scale = x.scale ? x.scale[adapter] : 1.0f;
        for (int ij = wave; ij < MB * NB; ij += WAVES) {
            const int i = ij / NB, j = ij % NB;
            const f32x4_t* const from = reinterpret_cast<const f32x4_t*>(lds4) + ij * 64 + lane;
            f32x4_t v = from[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v += from[w * (C::BYTES / 16)];
            const int r = r0 + j * 16 + kh * 4;
            if ((who >> (i * 16 + row) & 1) && r < x.rank) store_low(x, m0 + i * 16 + row, r, v * scale);
        }
        __syncthreads();
    }
}

template <int MB, int NB, int WAVES>
hipError_t launch_down(const LinearArgs& a, const AdapterArgs& x, int groups, hipStream_t s)
{
    constexpr int bytes = WAVES * SplitCfg<MB, NB, false>::BYTES;
    static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> told{0};
    const hipError_t e = allow_lds(&adapters_down_kernel<MB, NB, WAVES>, bytes, told);
    if (e != hipSuccess) return e;
    const long long list_tiles = x.tile ? ((long long)a.R + x.tile - 1) / x.tile : 0;
    const long long tiles = ((long long)a.R + MB * 16 - 1) / (MB * 16), blocks = (x.rank + NB * 16 - 1) / (NB * 16);
    const long long grid = (list_tiles + WAVES - 1) / WAVES + tiles * blocks * groups;
    hipLaunchKernelGGL((adapters_down_kernel<MB, NB, WAVES>), grid_of(grid), dim3(WAVES * 64), bytes, s, a, x, (int)list_tiles, groups);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adapters_down(const LinearArgs& a, const AdapterArgs& x, int, hipStream_t s)
{
    if (a.R <= 512) return launch_down<1, 1, 16>(a, x, 16, s);
    return launch_down<4, 4, 8>(a, x, 1, s);
}

hipError_t launch_linear_adapters(const LinearArgs& a, const AdapterArgs& x, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.N < 1 || a.K < 1 || a.w32 || x.n < 1 || x.rank < 8 || x.rank > kRankMost || x.rank % 8) return hipErrorInvalidValue;
    const int kernel = linear_kernel(a, n_cu);
    if (x.tile != linear_tile_rows(kernel)) return hipErrorInvalidValue;
    const hipError_t e = launch_adapters_down(a, x, n_cu, s);
    return e == hipSuccess ? launch_chosen(kernel, a, x, n_cu, s) : e;
}

}  // namespace moe_ep
